"""Workspaces of a decoder's layers: what is enough for the most rows and tokens is enough for fewer.  Launches are written down by a stand-in
for the HIP runtime (no GPU); the calls themselves refuse a workspace that is too small for what they would launch."""
import random

import pytest

from paper_1806_00588_amd import binding
from test_layers_launches import record          # noqa: F401  (a fixture)
from test_library_exports import _lib

MATRICES = [(1, 1, 32), (100, 300, 64), (1000, 1000, 128), (4096, 4096, 128), (8192, 8192, 64), (1000, 16384, 32), (64, 1 << 20, 128), (1 << 20, 128, 32), (40000, 1000, 32),
            (16384, 4096, 128), (33, 2304, 64)]
HEADS = [(16, 16, 128, 128), (4, 2, 64, 48), (1, 1, 16, 16), (20, 1, 256, 256), (12, 6, 96, 160)]


@pytest.mark.parametrize("N,K,group", MATRICES)
def test_packed_workspaces_never_fall(N, K, group):
    _lib()
    pp = binding.packed_params(N, K, group)
    sizes = [binding.packed_workspace_bytes(pp, M) for M in list(range(1, 1200)) + [1 << i for i in range(11, 17)]]
    assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("heads,k_heads,k_dim,v_dim", HEADS)
def test_delta_workspaces_never_fall(heads, k_heads, k_dim, v_dim):
    _lib()
    size = lambda S, B, T: binding.delta_workspace_bytes(binding.delta_params(S, B, T, heads, k_heads, k_dim, v_dim, 1.0))
    counts, tokens = [1, 2, 3, 5, 8, 9, 12, 16, 17, 26, 33, 64, 100, 256], [1, 2, 12, 13, 20, 21, 63, 64, 65, 128, 129, 1000, 8192]
    for T in tokens:
        for of in ([size(S, 1, T) for S in counts if S * T * heads <= 1 << 26], [size(2, B, T) for B in counts if 2 * B * T * heads <= 1 << 26]):
            assert of[0] > 0 and all(a <= b for a, b in zip(of, of[1:])), (T, of)
    for S in counts:
        of = [size(S, 3, T) for T in tokens if S * 3 * T * heads <= 1 << 26]       # (more is not supported, and has a size of 0)
        assert of[0] > 0 and all(a <= b for a, b in zip(of, of[1:])), (S, of)


def test_products_of_fewer_rows_in_the_most_rows_workspace(record):                            # noqa: F811
    rng = random.Random(2)
    calls = []
    for N, K, group in MATRICES:
        for most in (40, 128, 1000):
            room = binding.packed_workspace_bytes(binding.packed_params(N, K, group), most)
            for M in sorted({1, 15, 16, 17, 24, 25, 32, 33, 64, 65, 127, 128, 129, most} | {rng.randint(1, most) for _ in range(6)}):
                if M <= most:
                    calls += [(name, dict(N=N, K=K, group=group, M=M, x_type=x_type, x_ld=1 << 20, out_ld=1 << 24, bytes=room)) for name in ("linear", "gated") for x_type in (0, 1, 2)]
    bad = [(kw, got) for (_, kw), got in zip(calls, record(calls)) if got["status"] != 0]
    assert not bad, bad[:3]


def test_delta_rules_of_fewer_rows_and_tokens_in_the_most_workspace(record):                   # noqa: F811
    rng = random.Random(3)
    calls = []
    for heads, k_heads, k_dim, v_dim in HEADS:
        for S, T in ((9, 16), (64, 20), (26, 8192), (100, 300)):
            room = binding.delta_workspace_bytes(binding.delta_params(S, 1, T, heads, k_heads, k_dim, v_dim, 1.0))
            for s, t in [(1, T), (S, 1), (S, T), (min(S, 8), min(T, 16)), (S, min(T, 13))] + [(rng.randint(1, S), rng.randint(1, T)) for _ in range(10)]:
                calls += [("delta", dict(S=s, B=1, T=t, n_heads=heads, n_k_heads=k_heads, k_dim=k_dim, v_dim=v_dim, q_type=ty, k_type=ty, v_type=ty, out_type=ty,
                                         out_pitch=(t * heads * v_dim, heads * v_dim, v_dim), bytes=room)) for ty in (0, 1, 2)]
    bad = [(kw, got) for (_, kw), got in zip(calls, record(calls)) if got["status"] != 0]
    assert not bad, bad[:3]


@pytest.mark.parametrize("call", ["linear", "gated"])
def test_products_of_more_than_a_launch_has(record, call):                                     # noqa: F811
    """Refused before anything is launched, and no size is given for them; the largest that are not refused have one."""
    size = lambda kw: binding.packed_workspace_bytes(binding.packed_params(kw["N"], kw["K"], kw["group"]), kw["M"])
    of = lambda M, N, K, group=64: dict(N=N, K=K, group=group, M=M, x_ld=1 << 20, out_ld=1 << 24)
    too_many_rows, too_many_results, rows, results = of(1 << 20, 100, 1 << 20), of(1 << 20, 1 << 24, 128), of(1 << 20, 100, (1 << 17) - 128), of(1 << 14, 1 << 20, 128)
    assert size(too_many_rows) == 0 and all(size(kw) > 0 for kw in (too_many_results, rows, results))
    kinds = [dict(kw, x_type=ty, bytes=size(kw)) for kw in (too_many_rows, too_many_results, rows, results) for ty in (0, 1, 2)]
    assert [got["status"] for got in record([(call, kw) for kw in kinds])] == [2] * 6 + [0] * 6
