"""Plain references, in 64 bits, of a decoder's layers: weights of 4 bits and rows times them, the gated delta rule.  TEST
INFRASTRUCTURE: imported only by tests/; the product path never touches it.  numpy, from the definitions in include/lshbeam.h; no code is
shared with the HIP path."""
from __future__ import annotations

import math

import numpy as np


def place(n: int, k: int, parts: int):
    """(byte, upper four bits?) of the code of output n, input k in an array of codes; numbers or arrays."""
    tile, part, c = n // 16, k // 128, k % 32 // 8
    word, i = k % 128 // 32, k % 8
    return ((((tile * parts + part) * 4 + c) * 16 + n % 16) * 4 + word) * 4 + i % 4, i >= 4


def pack(codes: np.ndarray) -> np.ndarray:
    """codes [N, K] as they lie: uint8 [tiles, parts, 4, 16, 16], 0 behind the last."""
    N, K = codes.shape
    tiles, parts = -(-N // 16), -(-K // 128)
    out = np.zeros(tiles * parts * 1024, dtype=np.uint8)
    at, upper = place(np.arange(N)[:, None], np.arange(K)[None, :], parts)
    upper = np.broadcast_to(upper, at.shape)
    out[at[~upper]] = codes[~upper]              # (no two in one place)
    out[at[upper]] |= (codes[upper] << 4).astype(np.uint8)
    return out.reshape(tiles, parts, 4, 16, 16)


def unpack(packed: np.ndarray, N: int, K: int) -> np.ndarray:
    at, upper = place(np.arange(N)[:, None], np.arange(K)[None, :], packed.shape[1])
    return packed.reshape(-1)[at].astype(np.int64) >> 4 * upper & 15


def of_groups(x: np.ndarray, to_shape, fill=0):
    """[N, groups] numbers as scales and zeros lie: [tiles, parts, 16, 128 / group]."""
    out = np.full(to_shape, fill, dtype=x.dtype)
    n, g = np.arange(x.shape[0])[:, None], np.arange(x.shape[1])[None, :]
    out[n // 16, g // to_shape[3], n % 16, g % to_shape[3]] = x
    return out


def to_groups(x: np.ndarray, N: int, groups: int):
    n, g = np.arange(N)[:, None], np.arange(groups)[None, :]
    return x[n // 16, g // x.shape[3], n % 16, g % x.shape[3]]


def quantize(w: np.ndarray, group: int, round16, zeros: bool):
    """(codes [N, K], scales, zeros [N, groups]); round16: fp32 numbers to the scales' type and back."""
    N, K = w.shape
    groups = -(-K // group)
    codes, scales, zs = np.zeros((N, K), dtype=np.int64), np.zeros((N, groups)), np.zeros((N, groups), dtype=np.int64)
    for n in range(N):
        for g in range(groups):
            part = w[n, g * group:(g + 1) * group].astype(np.float64)
            if not np.isfinite(part).all():
                scales[n, g] = np.nan
                continue
            lo, hi = min(0.0, part.min()), max(0.0, part.max())
            with np.errstate(over="ignore"):
                s = float(round16(np.float32((hi - lo) / 15 if zeros else np.abs(part).max() / 7)))
            with np.errstate(invalid="ignore"):
                z = (min(15, max(0, int(np.rint(-lo / s)))) if s > 0 else 0) if zeros else 8
                q = np.rint(part / s) if s > 0 else np.zeros_like(part)
            codes[n, g * group:(g + 1) * group] = np.clip(q + z, 0, 15)
            scales[n, g], zs[n, g] = s, z
    return codes, scales, zs


def values(codes, scales, zeros, group: int):
    g = np.arange(codes.shape[1]) // group
    return (codes - zeros[:, g]) * scales[:, g]


def activation(x, name):
    if name == "silu":
        return x / (1 + np.exp(-x))
    if name == "gelu":
        return np.array([0.5 * v * math.erfc(-v / math.sqrt(2)) for v in x.reshape(-1)]).reshape(x.shape)
    return x / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))


def delta_rule(q, k, v, decay, beta, state, scale, n_new=None):
    """(out, state, size): q, k [R, T, Hk, Dk], v [R, T, H, Dv], state [R, H, Dk, Dv]; size [R, H, Dv]: the largest sum of the length of a
    state's column and |v| that a row came by.  Tokens behind n_new give zeros."""
    R, T, H, Dv = v.shape
    share = H // k.shape[2]
    S = state.astype(np.float64).copy()
    out = np.zeros((R, T, H, Dv))
    size = np.sqrt((S ** 2).sum(2))
    for r in range(R):
        for t in range(T if n_new is None else int(n_new[r])):
            for h in range(H):
                kk, qq = k[r, t, h // share].astype(np.float64), q[r, t, h // share].astype(np.float64)
                a = math.exp(float(decay[r, t, h]))
                u = float(beta[r, t, h]) * (v[r, t, h] - a * (kk @ S[r, h]))
                S[r, h] = a * S[r, h] + np.outer(kk, u)
                out[r, t, h] = scale * (qq @ S[r, h])
                size[r, h] = np.maximum(size[r, h], np.sqrt((S[r, h] ** 2).sum(0)) + np.abs(v[r, t, h]))
    return out, S, size
