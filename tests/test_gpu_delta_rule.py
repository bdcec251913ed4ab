"""lsh_delta_rule against a reference in 64 bits.

Tolerance: with keys of length 1, 0 <= beta <= 1 and decay <= 0 a token's map of the state never makes a column longer, so what a token's sums round
is carried on, not amplified.  A token rounds some k_dim + 64 times (its sums over the key, in chunks those over 64 tokens), by 2^-24 of the state's column
or the value; roundings of n tokens, of either sign, come to the root of their number, and 16 standard deviations are allowed:
2^-24 16 sqrt((n + 1) (k_dim + 64)) times the largest (length of the column + |v|) on the way.  A result is that times the length of the query and the
scale, and its own rounding."""
import numpy as np
import pytest

from oracle import layers
from test_gpu_packed import TYPES, half_step, in_64, on_gpu, torch_type, workspace

pytestmark = pytest.mark.gpu


def scene(rng, S, B, T, H, Hk, Dk, Dv, dtype, keys="random"):
    """Inputs as values that dtype has."""
    import torch
    R = S * B
    q, k = rng.normal(size=(2, R, T, Hk, Dk))
    if keys == "alike":                             # far from orthogonal: what one token wrote the next one takes away
        k = k * 0.2 + rng.normal(size=(R, 1, Hk, Dk))
    q, k = (x / np.sqrt((x ** 2).sum(-1, keepdims=True)) for x in (q, k))
    rate = np.exp(rng.random(H) * 5 - 3.5)
    decay = -rate * np.log1p(np.exp(rng.normal(size=(R, T, H)) - 2))
    beta = 1 / (1 + np.exp(-rng.normal(size=(R, T, H)) * 1.5))
    of = lambda x: torch.from_numpy(x).to(torch_type(dtype)).double().numpy()
    f32 = lambda x: x.astype(np.float32).astype(np.float64)
    return of(q), of(k), of(rng.normal(size=(R, T, H, Dv))), f32(decay), f32(beta), f32(rng.normal(size=(R, H, Dk, Dv)) * 0.3)


def check(rng, S, B, T, H, Hk, Dk, Dv, dtype, n_new=None, parents=None, fresh=False, in_place=False, fused=False, keys="random", scale=None):
    import torch
    from paper_1806_00588_amd import binding
    R = S * B
    q, k, v, decay, beta, state = scene(rng, S, B, T, H, Hk, Dk, Dv, dtype, keys)
    scale = Dk ** -0.5 if scale is None else scale
    begin = np.zeros_like(state) if fresh else state
    if parents is not None and not fresh:
        begin = np.stack([state[r // B * B + p] if 0 <= p < B else np.zeros_like(state[0]) for r, p in enumerate(parents)])
    n = np.full(R, T) if n_new is None else np.clip(n_new, 0, T)
    want, after, size = layers.delta_rule(q, k, v, decay, beta, begin, scale, n)
    if fused:                                       # views into one projection's results
        row = on_gpu(np.concatenate([x.reshape(R, T, -1) for x in (q, k, v)], 2), dtype)
        parts = row.split([Hk * Dk, Hk * Dk, H * Dv], 2)
        dq, dk, dv = (x.unflatten(2, (heads, -1)) for x, heads in zip(parts, (Hk, Hk, H)))
    else:
        dq, dk, dv = (on_gpu(x, dtype) for x in (q, k, v))
    dp = binding.delta_params(S, B, T, H, Hk, Dk, Dv, scale)
    before = None if fresh else on_gpu(state)
    to = before if in_place else torch.full((R, H, Dk, Dv), float("nan"), device="cuda")
    out = torch.full((R, T, H, Dv), 55.0, dtype=torch_type(dtype), device="cuda")
    if fused:
        out = torch.full((T, R, Dv, H + 1), 55.0, dtype=torch_type(dtype), device="cuda").permute(1, 0, 3, 2)[:, :, :H].contiguous()
    ws = workspace(binding.delta_workspace_bytes(dp))
    ws.fill_(255)
    i32 = lambda x: None if x is None else torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()
    binding.delta_rule(dp, dq, dk, dv, on_gpu(decay), on_gpu(beta), before, to, ws, out, parents=i32(parents), n_new=i32(n_new))
    tol = 2.0 ** -24 * 16 * np.sqrt((n + 1) * (Dk + 64))[:, None, None] * size          # [R, H, Dv]
    got = in_64(to)
    assert np.all(np.abs(got - after) <= tol[:, :, None]), (np.abs(got - after) / tol[:, :, None]).max()
    got = in_64(out)
    length = np.repeat(np.sqrt((q ** 2).sum(-1)), H // Hk, axis=2)[..., None] * abs(scale)
    for r in range(R):
        m = n[r]
        off = tol[r] * length[r, :m]
        assert np.all(np.abs(got[r, :m] - want[r, :m]) <= off + half_step(np.abs(want[r, :m]) + off, dtype))
        assert np.all(got[r, m:] == 55)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Dk,Dv", [(16, 16), (64, 64), (48, 80), (128, 128), (96, 160), (256, 32), (192, 256)])
def test_single_tokens(Dk, Dv, dtype):
    rng = np.random.default_rng(Dk + Dv)
    check(rng, 2, 3, 1, 4, 2, Dk, Dv, dtype, parents=[2, 0, 0, 1, 1, 1], fused=Dk == 48)
    check(rng, 3, 1, 1, 3, 3, Dk, Dv, dtype, in_place=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [2, 7, 8, 9, 16, 17, 31, 33])
def test_few_tokens(T, dtype):
    rng = np.random.default_rng(T)
    check(rng, 2, 2, T, 4, 2, 64, 48, dtype, n_new=[T, 0, 1, T - 1], parents=[1, 1, 0, -1])
    check(rng, 1, 1, T, 2, 1, 32, 64, dtype, fresh=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Dk,Dv", [(63, 64, 64), (64, 32, 48), (65, 128, 128), (128, 48, 16), (130, 96, 160), (200, 256, 80), (193, 16, 256), (400, 64, 32)])
def test_prompts(T, Dk, Dv, dtype):
    rng = np.random.default_rng(T + Dk)
    check(rng, 1, 3, T, 2, 1, Dk, Dv, dtype, n_new=[T, T // 2 + 1, 0], parents=[2, 0, 1], fused=T % 2 == 1)
    check(rng, 1, 1, T, 3, 3, Dk, Dv, dtype, fresh=True, keys="alike")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("S,H,Hk,T,Dk,Dv", [(30, 6, 2, 130, 32, 48), (9, 20, 20, 70, 64, 80), (50, 3, 1, 40, 16, 64), (17, 4, 4, 100, 128, 128), (6, 12, 3, 66, 192, 144),
                                            (11, 5, 5, 96, 256, 160)])
def test_many_rows_and_heads(S, H, Hk, T, Dk, Dv, dtype):
    """More workgroups than the chip takes at once: 32 columns each, some of them behind the last."""
    rng = np.random.default_rng(S + T)
    n_new = np.round(T * rng.random(S) ** 1.5).astype(int)
    n_new[-1] = T
    check(rng, S, 1, T, H, Hk, Dk, Dv, dtype, n_new=n_new)


@pytest.mark.parametrize("S,T", [(23, 200), (42, 130)])
def test_operands_that_take_turns_in_the_workspace(S, T):
    """460 and 840 pairs of a row and a head, a chunk's operands of 325 KB each: a chunk at a time, and a part of the pairs."""
    rng = np.random.default_rng(S)
    n_new = rng.integers(0, T + 1, S)
    n_new[:3] = T, 64, 65
    check(rng, S, 1, T, 20, 1, 256, 16, "f32", n_new=n_new, in_place=S == 23)
    check(rng, S // 2, 2, T, 20, 1, 256, 16, "f32", parents=rng.integers(-1, 2, S // 2 * 2))


@pytest.mark.parametrize("T", [1, 70])
def test_parents_and_counts_out_of_range(T):
    rng = np.random.default_rng(T)
    check(rng, 2, 3, T, 2, 2, 32, 32, "f32", n_new=[-5, T + 9, T, 1, 2 ** 31 - 1, -2 ** 31], parents=[3, -1, 2, 2 ** 31 - 1, -2 ** 31, 0])


@pytest.mark.parametrize("T", [1, 5, 90])
def test_in_place_and_scales(T):
    rng = np.random.default_rng(T)
    check(rng, 2, 1, T, 2, 2, 64, 64, "bf16", in_place=True, n_new=[T, 0], scale=-3.0)
    check(rng, 1, 1, T, 1, 1, 64, 64, "f32", scale=0.0)


@pytest.mark.parametrize("T", [1, 3, 100])
def test_many_beams_of_one_parent_and_many_heads(T):
    rng = np.random.default_rng(T)
    check(rng, 1, 12, T, 6, 2, 32, 32, "f16", parents=[5] * 12)
    check(rng, 1, 1, T, 24, 4, 16, 16, "bf16")


@pytest.mark.parametrize("T", [1, 6, 80])
def test_strong_and_no_decay(T):
    """Decays of 0 (nothing forgotten), of -200 (all of it), of -infinity."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(T)
    q, k, v, decay, beta, state = scene(rng, 1, 2, T, 2, 2, 32, 32, "f32")
    decay[0, :, 0], decay[0, :, 1], decay[1, T // 2, 0], decay[1, :, 1] = 0, -200, -np.inf, 0
    want, after, size = layers.delta_rule(q, k, v, decay, beta, state, 1.0)
    dp = binding.delta_params(1, 2, T, 2, 2, 32, 32, 1.0)
    to, out = torch.empty(2, 2, 32, 32, device="cuda"), torch.empty(2, T, 2, 32, device="cuda")
    binding.delta_rule(dp, *(on_gpu(x) for x in (q, k, v, decay, beta, state)), to, workspace(binding.delta_workspace_bytes(dp)), out)
    tol = 2.0 ** -24 * 16 * np.sqrt((T + 1) * 96) * size
    assert np.all(np.abs(in_64(to) - after) <= tol[:, :, None])
    assert np.all(np.abs(in_64(out) - want) <= tol[:, None])


@pytest.mark.parametrize("T", [1, 7, 150])
def test_beta_up_to_two_and_growing_states(T):
    """A beta of 2 turns a column round along the key, still not making it longer.  A decay of 0.02 makes it longer by e^(0.02 T) at most: what was rounded
    grows as the column itself does, whose largest length the tolerance has."""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(T)
    for grow in (False, True):
        q, k, v, decay, beta, state = scene(rng, 1, 2, T, 2, 2, 64, 48, "f32", keys="alike")
        beta = np.float32(beta * 2).astype(np.float64) if not grow else beta
        beta[0, :, 0] = 1 if grow else 2
        if grow:
            decay[:] = np.float32(0.02)
        want, after, size = layers.delta_rule(q, k, v, decay, beta, state, 1.0)
        dp = binding.delta_params(1, 2, T, 2, 2, 64, 48, 1.0)
        to, out = torch.empty(2, 2, 64, 48, device="cuda"), torch.empty(2, T, 2, 48, device="cuda")
        binding.delta_rule(dp, *(on_gpu(x) for x in (q, k, v, decay, beta, state)), to, workspace(binding.delta_workspace_bytes(dp)), out)
        tol = 2.0 ** -24 * 16 * np.sqrt((T + 1) * 128) * size
        assert np.all(np.abs(in_64(to) - after) <= tol[:, :, None])
        assert np.all(np.abs(in_64(out) - want) <= tol[:, None])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 9, 150])
def test_nothing_behind_the_last_token_is_used(T, dtype):
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(T)
    n_new = np.array([T, T // 2, 0, min(T, 65)])
    q, k, v, decay, beta, state = scene(rng, 4, 1, T, 2, 1, 48, 64, dtype)
    dp = binding.delta_params(4, 1, T, 2, 1, 48, 64, 1.0)
    ws, n, got = workspace(binding.delta_workspace_bytes(dp)), torch.from_numpy(n_new.astype(np.int32)).cuda(), []
    for bad in (False, True):
        for r in range(4):
            if bad:
                for x in (q, k, v, decay, beta):
                    x[r, n_new[r]:] = np.nan
        to, out = torch.zeros(4, 2, 48, 64, device="cuda"), torch.zeros(4, T, 2, 64, device="cuda", dtype=torch_type(dtype))
        binding.delta_rule(dp, *(on_gpu(x, dtype) for x in (q, k, v)), *(on_gpu(x) for x in (decay, beta, state)), to, ws, out, n_new=n)
        got.append((to, out))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and bool(torch.isfinite(got[1][0]).all())


@pytest.mark.parametrize("T", [1, 20, 150])
def test_rows_that_are_not_finite_are_alone(T):
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(T)
    q, k, v, decay, beta, state = scene(rng, 3, 1, T, 2, 1, 48, 64, "f32")
    dp = binding.delta_params(3, 1, T, 2, 1, 48, 64, 1.0)
    ws, got = workspace(binding.delta_workspace_bytes(dp)), []
    for bad in (False, True):
        if bad:
            v[1, T - 1, 0, 3], k[1, 0], state[1, 1, 2, 2] = np.nan, np.inf, np.nan
        to, out = torch.zeros(3, 2, 48, 64, device="cuda"), torch.zeros(3, T, 2, 64, device="cuda")
        binding.delta_rule(dp, *(on_gpu(x) for x in (q, k, v, decay, beta, state)), to, ws, out)
        got.append((to, out))
    for a, b in zip(*got):
        assert torch.equal(a[[0, 2]], b[[0, 2]]) and bool(torch.isfinite(a).all())


@pytest.mark.parametrize("T", [1, 12, 300])
def test_the_same_in_a_graph_and_on_another_stream(T):
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(T)
    dp = binding.delta_params(2, 2, T, 4, 2, 64, 64, 0.125)
    sets = [[on_gpu(x) for x in scene(rng, 2, 2, T, 4, 2, 64, 64, "f32")] for _ in range(2)]
    held = [torch.empty_like(x) for x in sets[0]]
    parents = torch.tensor([1, 0, 1, 1], dtype=torch.int32, device="cuda")
    ws, to, out = workspace(binding.delta_workspace_bytes(dp)), torch.empty(4, 4, 64, 64, device="cuda"), torch.empty(4, T, 4, 64, device="cuda")
    call = lambda: binding.delta_rule(dp, *held, to, ws, out, parents=parents)
    want = []
    for s in sets:
        for a, b in zip(held, s):
            a.copy_(b)
        call()
        want.append((to.clone(), out.clone()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(to, want[1][0]) and torch.equal(out, want[1][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(5):
        for a, b in zip(held, sets[turn % 2]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(to, want[turn % 2][0]) and torch.equal(out, want[turn % 2][1])
