"""What the GPU tests of a decoder's layers allow their results to be off in the mean is less than what a plane of bf16 that went missing costs: the operators in
64 bits with one of their numbers held in two planes instead of three."""
import numpy as np
import pytest

from test_gpu_delta_precision import allowed, keys
from test_gpu_packed_precision import rms


def bf16(x):
    u = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + (u >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)


def two_planes(x):
    first = bf16(x)
    return first + bf16(x - first)


@pytest.mark.parametrize("K", [128, 500, 2100])
@pytest.mark.parametrize("one_sign", [False, True])
def test_rows_of_fp32_in_two_planes(K, one_sign):
    rng = np.random.default_rng(K)
    x, w = rng.normal(size=(20, K)), rng.integers(-1, 2, (K, 300)) if one_sign else rng.integers(-8, 8, (K, 300))
    x = np.abs(x) if one_sign else x
    off, most = rms(two_planes(x) @ w - x @ w), 2.0 ** -24 * (1 + np.sqrt((K + -(-K // 32)) / 6)) * rms(x @ w)
    assert off > 2 * most, (off, most)


@pytest.mark.parametrize("Dk,entries", [(64, 64), (32, 16)])
@pytest.mark.parametrize("lost", [None, "state with k", "state with q", "both", "T", "V - K S", "A", "U", "U into the state"])
def test_a_chunk_with_a_number_in_two_planes(lost, Dk, entries):
    rng = np.random.default_rng(Dk)
    held = lambda name, x: two_planes(x) if lost == name or (lost == "both" and name.startswith("state")) else x
    k, S, v = keys(rng, (64,), Dk, entries, False), rng.normal(size=(Dk, 200)), rng.normal(size=(64, 200)) * 2.0 ** -12
    factor = float(np.float32(0.9))
    T = np.linalg.inv(np.eye(64) + np.tril(k @ k.T, -1))
    right = v - k @ held("state with k", S)
    u = held("T", T) @ held("V - K S", right)
    out = factor * k @ held("state with q", S) + held("A", factor * np.tril(k @ k.T)) @ held("U", u)
    state = S + k.T @ held("U into the state", u)
    off = max(rms(out - factor * v), rms(k[-1] @ state - v[-1]))
    assert (off > allowed(Dk, entries, False)) == (lost is not None), (off, allowed(Dk, entries, False))
