"""Rows times weights of 4 bits, how far results in fp32 are off in the mean: the root of the mean square of the errors over that of the results.

Tolerance: products x (code - zero) are exact.  A result adds up K of them and its groups' sums: K + groups roundings, each spread evenly over at most half a step of what has been added up,
2^-24 / sqrt(3) of it at most in the mean.  Terms are of random sign, so sums of i of them come to sqrt(i / K) of the result in the mean, and the squares of all these
roundings add up to (2^-24)^2 (K + groups) / 6 of the result's; its own last one, 2^-24, on top."""
import numpy as np
import pytest

from oracle import layers
from test_gpu_packed import TYPES, in_64, on_gpu, on_gpu_bytes, torch_type, workspace

pytestmark = pytest.mark.gpu


def rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


class Matrix:
    """Weights of 4 bits, on the GPU and as values.  near: codes next to their zeros, else anywhere."""

    def __init__(self, rng, N, K, group, zeros, near=False):
        import torch
        from paper_1806_00588_amd import binding
        tiles, parts, g = -(-N // 16), -(-K // 128), np.arange(K) // group
        self.N, self.K, self.group = N, K, group
        scales = (torch.from_numpy(np.exp(rng.normal(size=(N, g[-1] + 1)) * 0.5)) / np.sqrt(K)).half().double().numpy()
        offs = rng.integers(3, 13, (N, g[-1] + 1)) if zeros else np.full((N, g[-1] + 1), 8)
        codes = offs[:, g] + rng.integers(-1, 2, (N, K)) if near else rng.integers(0, 16, (N, K))
        self.values = layers.values(codes, scales, offs, group)
        shape = (tiles, parts, 16, 128 // group)
        self.pp = binding.packed_params(N, K, group)
        self.on_gpu = binding.PackedWeights(self.pp, codes=on_gpu_bytes(layers.pack(codes)), scales=on_gpu(layers.of_groups(scales, shape), "f16"),
                                            zeros=on_gpu_bytes(layers.of_groups(offs, shape)) if zeros else None)


def check(w, x, dtype):
    import torch
    from paper_1806_00588_amd import binding
    out = torch.empty(len(x), w.N, device="cuda")
    binding.packed_linear(w.pp, w.on_gpu, on_gpu(x, dtype), workspace(binding.packed_workspace_bytes(w.pp, len(x))), out)
    y = x @ w.values.T
    off, most = rms(in_64(out) - y) / rms(y), 2.0 ** -24 * (1 + np.sqrt((w.K + -(-w.K // w.group)) / 6))
    assert off <= most, (off, most)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 300, 128), (12, 200, 256), (12, 4500, 1000), (30, 300, 300), (40, 200, 6400), (130, 200, 520), (70, 17000, 2100)])
def test_rows_of_one_sign(M, N, K, group, zeros, dtype):
    """Behind an activation, say.  Codes are next to their zeros: the sum of codes as they are would be some sqrt(K) 8 times the result, and so would what is lost
    of it where the zeros are taken off afterwards."""
    import torch
    rng = np.random.default_rng(M + K + group)
    x = torch.from_numpy(np.abs(rng.normal(size=(M, K)))).to(torch_type(dtype)).double().numpy()
    check(Matrix(rng, N, K, group, zeros, near=True), x, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 300, 500), (12, 4500, 1000), (30, 300, 300), (40, 200, 6400), (130, 200, 520)])
def test_zeros_of_8_and_none(M, N, K, group, dtype):
    """Other conversions of the codes, the same results bit for bit, plain and gated (there also with one matrix of each)."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(M + K + group)
    x = on_gpu(rng.normal(size=(M, K)), dtype)
    none = [Matrix(rng, N, K, group, False) for _ in range(2)]
    pp, ws = none[0].pp, workspace(binding.packed_workspace_bytes(none[0].pp, M))
    eights = [binding.PackedWeights(pp, codes=w.on_gpu.codes, scales=w.on_gpu.scales, zeros=torch.full_like(w.on_gpu.scales, 8.0).to(torch.uint8)) for w in none]
    none = [w.on_gpu for w in none]
    outs = [torch.empty(M, N, device="cuda") for _ in range(6)]
    binding.packed_linear(pp, none[0], x, ws, outs[0])
    binding.packed_linear(pp, eights[0], x, ws, outs[1])
    for out, gate, up in zip(outs[2:], (none[0], eights[0], none[0], eights[0]), (none[1], eights[1], eights[1], none[1])):
        binding.packed_gated(pp, gate, up, x, ws, out)
    assert torch.equal(outs[0], outs[1]) and all(torch.equal(outs[2], out) for out in outs[3:])


@pytest.mark.parametrize("M,N,K", [(40, 100, 6400), (64, 17000, 2176), (129, 700, 128), (300, 270, 1024)])
def test_rows_of_bf16_from_where_they_lie(M, N, K):
    """Rows with a pitch of whole 16 bytes, with another one, and from an address between, have the same results bit for bit."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(M + K)
    w = Matrix(rng, N, K, 64, True)
    x = on_gpu(rng.normal(size=(M, K)), "bf16")
    check(w, in_64(x), "bf16")
    ws, outs = workspace(binding.packed_workspace_bytes(w.pp, M)), []
    for pitch, begin in ((0, 0), (24, 8), (3, 0), (8, 1)):
        held = torch.full((M, K + pitch), float("nan"), dtype=torch.bfloat16, device="cuda")
        held[:, begin:begin + K] = x
        outs.append(torch.empty(M, N, device="cuda"))
        binding.packed_linear(w.pp, w.on_gpu, held[:, begin:begin + K], ws, outs[-1])
    assert all(torch.equal(outs[0], out) for out in outs[1:])
