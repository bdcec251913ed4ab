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
