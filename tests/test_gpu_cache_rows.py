"""lsh_cache_attention where many rows of queries read the same keys, a wave for 16 of them: a row's own new tokens and query heads, and
beams over common blocks.  Tolerances as in test_gpu_cache.py, by the same arithmetic."""
import numpy as np
import pytest

from test_gpu_cache import check_attention, scene

pytestmark = pytest.mark.gpu


def own_rows(D, dtype, T, group):
    rng = np.random.default_rng(D + T)
    cp, pool, ref, tables, lengths = scene(rng, 5, 1, [0, 1, T, T + 1, 150 + T], 16, 1, D)
    check_attention(rng, cp, pool, ref, tables, lengths, dtype, T, group)


def common_rows(D, dtype, B, group):
    rng = np.random.default_rng(D + B)
    cp, pool, ref, tables, lengths = scene(rng, 2, B, [190 + 7 * (i % 23) for i in range(2 * B)], 16, 1, D, [176, 32], width=9000)
    check_attention(rng, cp, pool, ref, tables, lengths, dtype, 1, group, shared=np.array([11, 2]))


@pytest.mark.parametrize("D", [144, 208, 256])
@pytest.mark.parametrize("T,group", [(49, 1), (32, 2), (13, 5), (50, 4)])
def test_wide_heads_in_fp32(T, group, D):
    """49, 64, 65 and 200 rows: three planes of 64 rows would not fit in LDS beside two tiles."""
    own_rows(D, "f32", T, group)


@pytest.mark.parametrize("D", [144, 208, 256])
@pytest.mark.parametrize("B,group", [(7, 7), (16, 4), (13, 5), (25, 8)])
def test_wide_heads_in_fp32_over_common_blocks(B, group, D):
    common_rows(D, "f32", B, group)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [80, 128, 144, 192, 256])
@pytest.mark.parametrize("T,group", [(10, 4), (49, 1), (16, 4), (25, 4)])
def test_rows_of_every_head_size(T, group, D, dtype):
    """40, 49, 64 and 100 rows: three waves, four of them, two groups of four."""
    own_rows(D, dtype, T, group)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [80, 128, 144, 192, 256])
@pytest.mark.parametrize("B,group", [(8, 5), (7, 7), (16, 4), (25, 4), (6, 17)])
def test_rows_of_every_head_size_over_common_blocks(B, group, D, dtype):
    """The same, and (102 rows, 17 of a beam) with more than one wave for the beams' own parts too."""
    common_rows(D, dtype, B, group)


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,group,D", [(6, 1, 64), (6, 2, 80), (18, 2, 128), (18, 3, 48)])
def test_scales_that_are_not_finite_reach_only_who_sees_their_block(T, group, D, dtype, bad):
    """A block that some of a row's new tokens see and others do not: the last one, and with a window the first."""
    import torch
    from paper_1806_00588_amd import binding
    from test_gpu_cache import TYPES, ints, to_pool
    rng = np.random.default_rng(T + D)
    lengths = [48 + 2, 100, 64 + T - 1]        # (the last T positions of each lie in two blocks at least, or begin a tile's block)
    cp, _, ref, tables, lengths = scene(rng, 3, 1, lengths, 16, 1, D)
    q = torch.from_numpy(rng.standard_normal((3, T, group, D))).to(getattr(torch, TYPES[dtype])).cuda()
    td, ld = ints(tables), ints(lengths)
    for window, block in ((0, lambda r: (lengths[r] - 1) // 16), (33, lambda r: max(0, lengths[r] - T + 1 - 33) // 16)):
        ap = binding.attention_params(T, group, float(np.float32(1 / np.sqrt(D))), True, window)
        ws = torch.empty(binding.attention_workspace_bytes(cp, ap), dtype=torch.uint8, device="cuda")

        def run(pool):
            out = torch.empty_like(q)
            lse = torch.empty(3, T, group, device="cuda")
            binding.cache_attention(cp, ap, pool, q, td, ld, ws, out, lse=lse)
            torch.cuda.synchronize()
            return out, lse
        want = run(to_pool(cp, ref))
        assert all(bool(torch.isfinite(x).all()) for x in want)
        hurt = to_pool(cp, ref)
        hurt_keys = to_pool(cp, ref)
        for r in range(3):
            hurt.v_scale[tables[r, block(r)]] = bad
            hurt_keys.k_scale[tables[r, block(r)]] = bad
        out, lse = run(hurt)
        out_keys, lse_keys = run(hurt_keys)
        for r in range(3):
            lo, hi = 16 * block(r), 16 * block(r) + 16
            for t in range(T):
                end = lengths[r] - T + t + 1
                sees = end > lo and (not window or end - window < hi)
                assert torch.equal(lse[r, t], want[1][r, t])
                if not sees:
                    assert torch.equal(out[r, t], want[0][r, t]), (window, r, t)
                    assert torch.equal(out_keys[r, t], want[0][r, t]) and torch.equal(lse_keys[r, t], want[1][r, t])
                else:
                    assert not bool(torch.isfinite(out[r, t]).any()), (window, r, t)
            assert any(lengths[r] - T + t + 1 <= lo or (window and lengths[r] - T + t + 1 - window >= hi) for t in range(T))
