"""A decoder's layers on memory whose offsets pass 32 bits: rows, results, states and codes gigabytes apart.  Every call is made once more on
memory close together, with the same results bit for bit; of codes beyond 4 GiB some outputs are compared with the reference."""
import numpy as np
import pytest

from oracle import layers
from test_gpu_delta_rule import scene
from test_gpu_packed import Weights, half_step, in_64, on_gpu, rows_of, torch_type, workspace

pytestmark = pytest.mark.gpu

FAR = (1 << 31) + 2000                     # elements


def far_rows(x):
    """The same values, rows FAR elements apart (uninitialised memory between them)."""
    import torch
    big = torch.empty((x.shape[0] - 1) * FAR + x.shape[1], dtype=x.dtype, device="cuda")
    view = big.as_strided(tuple(x.shape), (FAR, 1))
    view.copy_(x)
    return view


@pytest.mark.parametrize("M", [3, 150])
def test_rows_and_results_far_apart(M):
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(M)
    w, up = Weights(rng, 200, 300, 64), Weights(rng, 200, 300, 64, zeros=True)
    x = on_gpu(rows_of(rng, M, 300, "bf16"), "bf16")
    ws = workspace(binding.packed_workspace_bytes(w.pp, M))
    near = [torch.empty(M, 200, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    binding.packed_linear(w.pp, w.on_gpu, x, ws, near[0], add=x[:, :200])
    binding.packed_gated(w.pp, w.on_gpu, up.on_gpu, x, ws, near[1])
    if M > 3:                              # (that many rows do not fit so far apart: the last of them)
        pitch = FAR // 64
        big = torch.empty((M - 1) * pitch + 300, dtype=torch.bfloat16, device="cuda")
        fx = big.as_strided((M, 300), (pitch, 1))
        fx.copy_(x)
        out = torch.empty((M - 1) * pitch + 200, dtype=torch.bfloat16, device="cuda").as_strided((M, 200), (pitch, 1))
    else:
        fx, out = far_rows(x), far_rows(near[0])
    binding.packed_linear(w.pp, w.on_gpu, fx, ws, out, add=fx[:, :200])
    assert torch.equal(out, near[0])
    binding.packed_gated(w.pp, w.on_gpu, up.on_gpu, fx, ws, out)
    assert torch.equal(out, near[1])


def test_weights_far_apart():
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(2)
    x = on_gpu(rng.normal(size=(3, 300)), "bf16")
    pp = binding.packed_params(3, 300, 32)
    a, b = (binding.PackedWeights(pp, zeros=True) for _ in range(2))
    binding.packed_quantize(pp, x, a)
    far = far_rows(x)
    binding.packed_quantize(pp, far, b)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales) and torch.equal(a.zeros, b.zeros)
    out = torch.empty(3, 300, dtype=torch.bfloat16, device="cuda")
    binding.packed_values(pp, a, out)
    binding.packed_values(pp, a, far)
    assert torch.equal(out, far)


@pytest.mark.parametrize("M", [2, 40])
def test_codes_beyond_4_gib(M):
    import torch
    from paper_1806_00588_amd import binding
    N, K, group = (1 << 21) + 8, 4200, 128
    tiles, parts = -(-N // 16), -(-K // 128)
    pp = binding.packed_params(N, K, group)
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.empty(tiles, parts, 4, 16, 16, dtype=torch.uint8, device="cuda")
    codes.view(-1).view(torch.int32).random_(generator=g)
    scales = (torch.rand(tiles, parts, 16, 1, device="cuda", generator=g) + 0.5).to(torch.float16) / 64
    assert codes.numel() > 1 << 32
    w = binding.PackedWeights(pp, codes=codes, scales=scales)
    rng = np.random.default_rng(M)
    x = rows_of(rng, M, K, "f16")
    out = torch.empty(M, N, device="cuda")
    binding.packed_linear(pp, w, on_gpu(x, "f16"), workspace(binding.packed_workspace_bytes(pp, M)), out)
    for tile in (0, tiles // 2, (1 << 32) // (parts * 1024), tiles - 2):
        c = layers.unpack(codes[tile:tile + 2].cpu().numpy(), 32, K)
        s = layers.to_groups(in_64(scales[tile:tile + 2]), 32, parts)
        values = layers.values(c, s, np.full_like(s, 8), group)
        sizes = layers.values(c, s, np.full_like(s, -8), group)
        n = min(32, N - 16 * tile)
        y, off = x @ values[:n].T, (group + parts + 12) * 2.0 ** -23 * (np.abs(x) @ sizes[:n].T)
        got = in_64(out[:, 16 * tile:16 * tile + n])
        assert np.all(np.abs(got - y) <= off + half_step(np.abs(y) + off, "f32")), tile


@pytest.mark.parametrize("T", [1, 6, 70])
def test_tokens_and_states_far_apart(T):
    """Rows of queries, keys, values and results FAR elements apart; states of 65536 pairs of 128 x 128 are 4 GiB."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(T)
    args = [on_gpu(x, "bf16" if i < 3 else "f32") for i, x in enumerate(scene(rng, 2, 1, T, 4, 2, 32, 48, "bf16"))]
    dp = binding.delta_params(2, 1, T, 4, 2, 32, 48, 1.0)
    ws = workspace(binding.delta_workspace_bytes(dp))

    def far(x):
        view = torch.empty(FAR + x[0].numel(), dtype=x.dtype, device="cuda").as_strided(tuple(x.shape), (FAR,) + tuple(x.stride()[1:]))
        view.copy_(x)
        return view

    results = []
    for place in (lambda x: x, far):
        q, k, v = (place(x) for x in args[:3])
        out, to = place(torch.zeros(2, T, 4, 48, dtype=torch.bfloat16, device="cuda")), torch.empty(2, 4, 32, 48, device="cuda")
        binding.delta_rule(dp, q, k, v, args[3], args[4], args[5], to, ws, out)
        results.append((out.clone(), to))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])


@pytest.mark.parametrize("T", [1, 2, 33])
def test_states_beyond_4_gib(T):
    """The last row of many continues as it does alone."""
    import torch
    from paper_1806_00588_amd import binding
    R, H, D = 1100, 64, 128
    rng = np.random.default_rng(T)
    q, k, v, decay, beta, state = (on_gpu(x) for x in scene(rng, 1, 1, T, H, H, D, D, "f32"))
    n_new = torch.zeros(R, dtype=torch.int32, device="cuda")
    n_new[-1] = T
    states = torch.zeros(R, H, D, D, device="cuda")
    assert states.numel() * 4 > 1 << 32
    states[-1] = state[0]
    spread = lambda x: x.expand((R,) + tuple(x.shape[1:]))
    dp = binding.delta_params(R, 1, T, H, H, D, D, 1.0)
    out = torch.zeros(R, T, H, D, device="cuda")
    binding.delta_rule(dp, spread(q), spread(k), spread(v), spread(decay).contiguous(), spread(beta).contiguous(), states, states,
                       workspace(binding.delta_workspace_bytes(dp)), out, n_new=n_new)
    alone = binding.delta_params(1, 1, T, H, H, D, D, 1.0)
    want, to = torch.empty(1, T, H, D, device="cuda"), torch.empty(1, H, D, D, device="cuda")
    binding.delta_rule(alone, q, k, v, decay, beta, state, to, workspace(binding.delta_workspace_bytes(alone)), want)
    tol = 2.0 ** -24 * 16 * np.sqrt((T + 1) * (D + 64)) * 40       # (as in test_gpu_delta_rule.py; no column's length and value come to 40)
    assert bool(((states[-1] - to[0]).abs() <= tol).all()) and bool(((out[-1] - want[0]).abs() <= tol).all())
    assert not bool(states[:-1].any()) and not bool(out[:-1].any())
