"""Many rows times weights of 4 bits where a workgroup has 128 rows: sizes whose plan takes those kernels (test_layers_kernels.py says which each takes).

Tolerance: every product x (code - zero) is exact, and K + groups sums, what is added, and the bias round by 2^-24 each, of no more than
sum |x| |code - zero| scale + |bias| + |add|.  Of a gated result as in test_gpu_packed.py.  In the mean as in test_gpu_packed_precision.py."""
import numpy as np
import pytest

from oracle import layers
from test_gpu_packed import TYPES, half_step, in_64, on_gpu, rows_of, torch_type, workspace
from test_gpu_packed_precision import Matrix, rms

pytestmark = pytest.mark.gpu

# M, N, K, (type, group) for which they are
LINEAR = [(2050, 1000, 300, [(t, g) for t in TYPES for g in (32, 64, 128)]), (2050, 1000, 1152, [(t, 64) for t in TYPES]),
          (777, 5000, 300, [("bf16", 64), ("bf16", 128), ("f16", 64), ("f16", 128)]), (777, 5000, 256, [("bf16", 64), ("bf16", 128), ("f16", 64), ("f16", 128)]),
          (1500, 4100, 300, [("f32", 64), ("f32", 128)]), (1500, 4100, 1100, [("f32", 128), ("bf16", 128)])]
GATED = [(2050, 500, 300, [(t, g) for t in TYPES for g in (32, 64, 128)]), (2050, 1000, 300, [("bf16", 64), ("bf16", 128), ("f16", 64), ("f16", 128)]),
         (2050, 1000, 256, [("bf16", 64), ("f16", 128)]), (1030, 3000, 300, [("f32", 64), ("f32", 128)]), (1030, 3000, 1100, [("f32", 64), ("f16", 64)])]
flat = lambda cases: [(M, N, K, group, dtype) for M, N, K, kinds in cases for dtype, group in kinds]


def bound(w, x):
    return (w.K + -(-w.K // w.group) + 2) * 2.0 ** -24 * (np.abs(x) @ np.abs(w.values.T))


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,N,K,group,dtype", flat(LINEAR))
def test_linear(M, N, K, group, dtype, zeros):
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(M + K + group)
    w, x = Matrix(rng, N, K, group, zeros), rows_of(rng, M, K, dtype)
    ws, out = workspace(binding.packed_workspace_bytes(w.pp, M)), torch.full((M, N + 3), 77.0, device="cuda")
    binding.packed_linear(w.pp, w.on_gpu, on_gpu(x, dtype), ws, out[:, :N])
    y, off = x @ w.values.T, bound(w, x)
    got = in_64(out[:, :N])
    assert np.all(np.abs(got - y) <= off + half_step(np.abs(y) + off, "f32")) and bool((out[:, N:] == 77).all())
    assert rms(got - y) <= 2.0 ** -24 * (1 + np.sqrt((K + -(-K // group)) / 6)) * rms(y)
    # with a bias and on top of what is there, in the rows' type
    b, more = rng.normal(size=N).astype(np.float32), on_gpu(rng.normal(size=(M, N)), dtype)
    y, off = y + b + in_64(more), off + 3 * 2.0 ** -24 * (np.abs(b) + np.abs(in_64(more)))
    binding.packed_linear(w.pp, w.on_gpu, on_gpu(x, dtype), ws, more, bias=on_gpu(b), add=more)
    assert np.all(np.abs(in_64(more) - y) <= off + half_step(np.abs(y) + off, dtype))


@pytest.mark.parametrize("zeros", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("M,N,K,group,dtype", flat(GATED))
def test_gated(M, N, K, group, dtype, zeros):
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(M + K + group)
    (gate, up), x = (Matrix(rng, N, K, group, z) for z in zeros), rows_of(rng, M, K, dtype)
    out = torch.empty(M, N, device="cuda")
    binding.packed_gated(gate.pp, gate.on_gpu, up.on_gpu, on_gpu(x, dtype), workspace(binding.packed_workspace_bytes(gate.pp, M)), out)
    g, u, g_off, u_off = x @ gate.values.T, x @ up.values.T, bound(gate, x), bound(up, x)
    a = layers.activation(g, "silu")
    a_off = 1.13 * g_off + 2.0 ** -20 * np.abs(a) + 2.0 ** -22
    want, off = a * u, a_off * (np.abs(u) + u_off) + np.abs(a) * u_off
    assert np.all(np.abs(in_64(out) - want) <= off + half_step(np.abs(want) + off, "f32"))
