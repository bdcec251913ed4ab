"""lsh_delta_rule by every kernel that is built for it (test_layers_kernels.py says that none is left out), on operands and results with pitches of their own: heads, tokens and rows
in any order, gaps between heads that are no multiple of anything.  Tolerances as in test_gpu_delta_rule.py."""
import numpy as np
import pytest

from oracle import layers
from test_gpu_delta_rule import scene
from test_gpu_packed import TYPES, half_step, in_64, on_gpu, torch_type, workspace

pytestmark = pytest.mark.gpu

# S, H, Hk, T, Dk, Dv: single tokens and a few, by the rows of the state that a thread has; chunks, by k_dim; these with more than 512 workgroups of 16 columns
FEW = [(2, 4, 2, T, Dk, Dv) for T in (1, 5) for Dk, Dv in ((16, 48), (48, 64), (96, 32), (112, 80), (160, 16), (208, 144))]
CHUNKS = [(2, 2, 1, 70, Dk, Dv) for Dk, Dv in ((32, 48), (64, 16), (80, 64), (128, 32), (160, 96), (240, 48))]
MANY = [(18, 4, 2, 66, Dk, Dv) for Dk, Dv in ((16, 128), (48, 144), (96, 128), (112, 128), (176, 128), (256, 144))]


def spread(x, order, gap, dtype, fill):
    """[R, T, heads, D] with its dimensions in another order in memory, `gap` elements behind each head; the memory, and x in it."""
    import torch
    back = [order.index(i) for i in range(3)] + [3]
    held = torch.full([x.shape[i] for i in order] + [x.shape[3] + gap], fill, dtype=torch_type(dtype), device="cuda")
    view = held.permute(back)[..., :x.shape[3]]
    view.copy_(on_gpu(x, dtype))
    return held, view


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("S,H,Hk,T,Dk,Dv", FEW + CHUNKS + MANY)
def test_every_kernel(S, H, Hk, T, Dk, Dv, dtype):
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(Dk + T)
    q, k, v, decay, beta, state = scene(rng, S, 1, T, H, Hk, Dk, Dv, dtype)
    n = np.maximum(1, np.round(T * rng.random(S) ** 0.5)).astype(int)
    n[-1] = T
    want, after, size = layers.delta_rule(q, k, v, decay, beta, state, Dk ** -0.5, n)
    _, dq = spread(q, (0, 1, 2), 3, dtype, np.nan)
    _, dk = spread(k, (2, 0, 1), 5, dtype, np.nan)
    _, dv = spread(v, (0, 2, 1), 8, dtype, np.nan)
    held, out = spread(np.full(v.shape, 55.0), (1, 2, 0), 7, dtype, 55.0)
    dp = binding.delta_params(S, 1, T, H, Hk, Dk, Dv, Dk ** -0.5)
    to, ws = torch.empty(S, H, Dk, Dv, device="cuda"), workspace(binding.delta_workspace_bytes(dp))
    binding.delta_rule(dp, dq, dk, dv, on_gpu(decay), on_gpu(beta), on_gpu(state), to, ws, out, n_new=torch.from_numpy(n.astype(np.int32)).cuda())
    tol = 2.0 ** -24 * 16 * np.sqrt((n + 1) * (Dk + 64))[:, None, None] * size
    assert np.all(np.abs(in_64(to) - after) <= tol[:, :, None])
    got, length = in_64(out), np.repeat(np.sqrt((q ** 2).sum(-1)), H // Hk, axis=2)[..., None] * Dk ** -0.5
    for r in range(S):
        off = tol[r] * length[r, :n[r]]
        assert np.all(np.abs(got[r, :n[r]] - want[r, :n[r]]) <= off + half_step(np.abs(want[r, :n[r]]) + off, dtype))
        assert np.all(got[r, n[r]:] == 55)
    assert bool((held[..., Dv:] == 55).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,at", [(1, 0), (9, 4), (150, 100)])
def test_heads_that_are_not_finite_are_alone(T, at, dtype):
    """Row 1: a NaN in a value of head 0, an infinity in the second key head's keys (heads 2 and 3), the first at token `at`.  Head 1, with the first
    head's keys, and other columns of head 0 are as without them; what they reach is not finite from that token on, and as without them before its chunk."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(T)
    q, k, v, decay, beta, state = scene(rng, 3, 1, T, 4, 2, 48, 64, dtype)
    dp = binding.delta_params(3, 1, T, 4, 2, 48, 64, 1.0)
    ws, got = workspace(binding.delta_workspace_bytes(dp)), []
    for bad in (False, True):
        if bad:
            v[1, at, 0, 3], k[1, at, 1, 7] = np.nan, np.inf
        to, out = torch.zeros(3, 4, 48, 64, device="cuda"), torch.zeros(3, T, 4, 64, device="cuda", dtype=torch_type(dtype))
        binding.delta_rule(dp, *(on_gpu(x, dtype) for x in (q, k, v)), *(on_gpu(x) for x in (decay, beta, state)), to, ws, out)
        got.append((to, out))
    (to, out), (bad_to, bad_out) = got
    columns = [c for c in range(64) if c != 3]
    assert torch.equal(to[[0, 2]], bad_to[[0, 2]]) and torch.equal(out[[0, 2]], bad_out[[0, 2]])
    assert torch.equal(to[1, 1], bad_to[1, 1]) and torch.equal(out[1, :, 1], bad_out[1, :, 1])
    assert torch.equal(to[1, 0][:, columns], bad_to[1, 0][:, columns]) and torch.equal(out[1, :, 0][:, columns], bad_out[1, :, 0][:, columns])
    assert torch.equal(out[1, :at // 64 * 64], bad_out[1, :at // 64 * 64])
    assert not bool(torch.isfinite(bad_to[1, 0, :, 3]).any()) and not bool(torch.isfinite(bad_out[1, at:, 0, 3]).any())
    assert not bool(torch.isfinite(bad_to[1, 2:]).any()) and not bool(torch.isfinite(bad_out[1, at:, 2:]).any())
