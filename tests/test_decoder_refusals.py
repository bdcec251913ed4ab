"""Calls that the selection from logits and the cache's operators refuse, through the C ABI and without a GPU: arguments are
looked at before anything is launched.  Pointers are made up; none is followed."""
import ctypes

import pytest

from paper_1806_00588_amd import binding
from test_library_exports import _lib

INVALID, UNSUPPORTED, SMALL = 1, 2, 6
P = 1 << 20                        # an address at a multiple of 256
BIG = 1 << 40


def _select(**kw):
    a = dict(S=2, B=3, N=3, V=100, dtype=0, ld=100, allowed_ld=0, logits=P, scores=P, allowed=None, ws=P, bytes=BIG, beam=P, word=P, score=P,
             lse=None)
    a.update(kw)
    p = binding.SelectParams(a["S"], a["B"], a["N"], a["V"], a["dtype"], a["ld"], a["allowed_ld"])
    return _lib().lsh_beam_select(ctypes.byref(p), a["logits"], a["scores"], a["allowed"], a["ws"], a["bytes"], a["beam"], a["word"],
                                  a["score"], a["lse"], None)


@pytest.mark.parametrize("kw", [
    {"S": 0}, {"S": -1}, {"B": 0}, {"B": 257}, {"N": 0}, {"N": 257}, {"V": 0}, {"V": (1 << 24) + 1, "ld": 1 << 25}, {"S": 1 << 20}, {"dtype": 3},
    {"dtype": -1}, {"ld": 99}, {"logits": None}, {"logits": P + 2}, {"logits": P + 1, "dtype": 1}, {"scores": None}, {"ws": None}, {"ws": P + 16},
    {"beam": None}, {"word": None}, {"score": None}, {"allowed": P, "allowed_ld": 3}, {"allowed": P, "allowed_ld": -4}],
    ids=lambda k: ",".join("%s=%s" % i for i in k.items()))
def test_select_refuses(kw):
    assert _select(**kw) == INVALID


def test_select_workspace():
    lib = _lib()
    p = binding.select_params(2, 3, 70000)
    n = binding.select_workspace_bytes(p)
    assert n >= 6 * (70000 // 128) * 4
    assert _select(V=70000, ld=70000, bytes=n - 1) == SMALL
    assert binding.select_workspace_bytes(binding.select_params(2, 300, 10)) == 0
    assert lib.lsh_select_workspace_bytes(None) == 0
    assert lib.lsh_beam_select(None, P, P, None, P, BIG, P, P, P, None, None) == INVALID


CACHE = dict(S=2, B=3, n_blocks=50, block=16, max_blocks=10, n_heads=2, head_dim=64)
BAD_CACHES = [{"S": 0}, {"B": 0}, {"B": 257}, {"S": 1 << 20}, {"n_blocks": 0}, {"n_blocks": (1 << 24) + 1}, {"n_blocks": 1 << 24, "block": 128},
              {"block": 0}, {"block": 8}, {"block": 24}, {"block": 256}, {"max_blocks": 0}, {"max_blocks": (1 << 20) + 1}, {"n_heads": 0},
              {"n_heads": 65536}, {"head_dim": 0}, {"head_dim": 8}, {"head_dim": 72}, {"head_dim": 272}]


def _cache(**kw):
    a = dict(CACHE)
    a.update({k: v for k, v in kw.items() if k in CACHE})
    return binding.cache_params(**a)


def _advance(**kw):
    a = dict(T=1, parents=None, n_new=None, tables_in=P, lengths_in=P, tables_out=2 * P, lengths_out=2 * P, slots=P, copy_from=P, shared=None,
             status=P, ws=P, bytes=BIG)
    a.update({k: v for k, v in kw.items() if k not in CACHE})
    return _lib().lsh_cache_advance(ctypes.byref(_cache(**kw)), a["T"], a["parents"], a["n_new"], a["tables_in"], a["lengths_in"], a["tables_out"],
                                    a["lengths_out"], a["slots"], a["copy_from"], a["shared"], a["status"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw", BAD_CACHES + [{"T": 0}, {"T": -1}, {"tables_in": None}, {"lengths_in": None}, {"tables_out": None},
                                             {"lengths_out": None}, {"tables_out": P}, {"lengths_out": P}, {"slots": None}, {"copy_from": None},
                                             {"status": None}, {"ws": None}, {"ws": P + 64}], ids=lambda k: ",".join("%s=%s" % i for i in k.items()))
def test_advance_refuses(kw):
    assert _advance(**kw) == INVALID


def test_advance_workspace():
    n = binding.cache_workspace_bytes(_cache())
    assert n > 0 and _advance(bytes=n - 1) == SMALL
    assert all(binding.cache_workspace_bytes(_cache(**kw)) == 0 for kw in BAD_CACHES)
    assert _lib().lsh_cache_workspace_bytes(None) == 0
    assert _lib().lsh_cache_advance(None, 1, *[P] * 11, BIG, None) == INVALID


def _pool(k=P, v=P, k_scale=P, v_scale=P):
    return binding._PoolPointers(k, v, k_scale, v_scale)


def _write(**kw):
    a = dict(T=1, pool=_pool(), k=P, v=P, k_type=0, v_type=0, pitch=64, slots=P, copy_from=None)
    a.update({k: v for k, v in kw.items() if k not in CACHE})
    kr, vr = binding._Rows(a["k_type"], 128, 128, a["pitch"]), binding._Rows(a["v_type"], 128, 128, 64)
    return _lib().lsh_cache_write(ctypes.byref(_cache(**kw)), ctypes.byref(a["pool"]), a["T"], a["k"], ctypes.byref(kr), a["v"], ctypes.byref(vr),
                                  a["slots"], a["copy_from"], None)


BAD_POOLS = [{"pool": _pool(k=None)}, {"pool": _pool(v=None)}, {"pool": _pool(k_scale=None)}, {"pool": _pool(v_scale=None)}, {"pool": _pool(k=P + 8)},
             {"pool": _pool(v=P + 8)}]


@pytest.mark.parametrize("kw", BAD_CACHES + BAD_POOLS + [{"T": 0}, {"k": None}, {"v": None}, {"slots": None}, {"k_type": 1}, {"v_type": 2},
                                                         {"k_type": 3, "v_type": 3}, {"pitch": -64}, {"k": P + 2}, {"v": P + 2}],
                         ids=lambda k: ",".join("%s=%s" % (a, b if isinstance(b, (int, type(None))) else "bad") for a, b in k.items()))
def test_write_refuses(kw):
    assert _write(**kw) == INVALID


def test_write_refuses_more_workgroups_than_a_launch_has():
    assert _write(S=1 << 12, B=256, T=1 << 10) == UNSUPPORTED


def _attention(**kw):
    a = dict(T=1, q_heads=4, causal=1, window=0, scale=1.0, pool=_pool(), q=P, q_type=0, out_type=0, tables=P, lengths=P, n_new=None, shared=None,
             ws=P, bytes=BIG, out=P, lse=None, out_pitch=(256, 256, 64))
    a.update({k: v for k, v in kw.items() if k not in CACHE})
    p = binding.AttentionParams(a["T"], a["q_heads"], a["causal"], a["window"], a["scale"])
    qr, orow = binding._Rows(a["q_type"], 256, 256, 64), binding._Rows(a["out_type"], *a["out_pitch"])
    return _lib().lsh_cache_attention(ctypes.byref(_cache(**kw)), ctypes.byref(a["pool"]), ctypes.byref(p), a["q"], ctypes.byref(qr), a["tables"],
                                      a["lengths"], a["n_new"], a["shared"], a["ws"], a["bytes"], a["out"], ctypes.byref(orow), a["lse"], None)


@pytest.mark.parametrize("kw", BAD_CACHES + BAD_POOLS + [
    {"T": 0}, {"q_heads": 0}, {"q_heads": 3}, {"q_heads": 1 << 17}, {"window": -1}, {"window": 5, "causal": 0}, {"scale": 0.0}, {"scale": -1.0},
    {"scale": float("inf")}, {"scale": float("nan")}, {"q": None}, {"q": P + 2}, {"tables": None}, {"lengths": None}, {"out": None}, {"q_type": 1},
    {"q_type": 5, "out_type": 5}, {"ws": None}, {"ws": P + 128}],
    ids=lambda k: ",".join("%s=%s" % (a, b if isinstance(b, (int, float, type(None))) else "bad") for a, b in k.items()))
def test_attention_refuses(kw):
    assert _attention(**kw) == INVALID


def test_attention_workspace():
    lib = _lib()
    n = binding.attention_workspace_bytes(_cache(), binding.attention_params(1, 4, 1.0))
    assert n > 0 and _attention(bytes=n - 1) == SMALL
    assert binding.attention_workspace_bytes(_cache(), binding.attention_params(1, 3, 1.0)) == 0
    assert binding.attention_workspace_bytes(_cache(block=24), binding.attention_params(1, 4, 1.0)) == 0
    assert lib.lsh_attention_workspace_bytes(None, None) == 0
    assert _attention(S=1 << 12, B=256, T=1 << 10) == UNSUPPORTED


def test_a_pool_of_host_tensors_is_refused():
    import torch
    with pytest.raises(ValueError):
        binding.CachePool(_cache(), k=torch.zeros(50, 2, 4, 16, 16, dtype=torch.uint8))


@pytest.mark.parametrize("kw", [
    dict(S=1, B=256, n_blocks=1000, max_blocks=1000, n_heads=1, T=1 << 20, q_heads=1024),      # groups of 64 rows: 2^32
    dict(S=1, B=256, n_blocks=1000, max_blocks=1000, n_heads=1, T=1 << 20, q_heads=1025),
    dict(S=1 << 20, B=1, n_heads=65535, T=1 << 20, q_heads=65535), dict(S=1, B=1, T=1 << 20, q_heads=65534), dict(S=1, B=1, T=1 << 20, q_heads=66)],
    ids=lambda k: ",".join("%s=%s" % i for i in k.items()))
def test_attention_of_too_many_rows(kw):
    """Numbers of rows that no launch has, and whose groups and workgroups pass 32 or 64 bits."""
    assert _attention(**kw) == UNSUPPORTED and _attention(shared=P, **kw) == UNSUPPORTED
    assert binding.attention_workspace_bytes(_cache(**kw), binding.attention_params(kw["T"], kw["q_heads"], 1.0)) == 0


def test_attention_workspace_of_many_rows_goes_with_the_call():
    """Up to the last supported call the workspace has a size, and a byte less than that is too little."""
    for kw in (dict(S=1, B=1, T=1 << 20, q_heads=62), dict(S=1 << 12, B=256, T=1, q_heads=10), dict(S=1, B=256, T=1 << 12, q_heads=62)):
        n = binding.attention_workspace_bytes(_cache(**kw), binding.attention_params(kw["T"], kw["q_heads"], 1.0))
        assert n > 0 and _attention(bytes=n - 1, out_pitch=side_by_side(kw["T"], kw["q_heads"], 64), **kw) == SMALL


def test_select_takes_as_many_results_as_its_sentences_may_have():
    """S * B is bounded, S * N is not: 2^20 sentences of a beam can have 256 results each."""
    for S, N in ((8192, 200), (1 << 20, 256)):
        n = binding.select_workspace_bytes(binding.select_params(S, 1, 100, N))
        assert n > 0 and _select(S=S, B=1, N=N, bytes=n - 1) == SMALL


@pytest.mark.parametrize("T", [(1 << 27) + 1, (1 << 31) - 256, (1 << 31) - 1])
def test_more_new_tokens_than_any_table_holds(T):
    """2^20 blocks of 128 tokens are the most; counting beyond 2^31 by a workgroup's threads would pass 32 bits."""
    assert _advance(T=T) == INVALID
    assert _write(T=T) == INVALID and _write(T=T, block=128) == INVALID


def side_by_side(T, heads, D):
    """Pitches of rows, tokens and heads with nothing between them."""
    return T * heads * D, heads * D, D


def _places(R, T, H, D, pitch):
    """Whether heads lie on each other, by writing down every place."""
    at = [r * pitch[0] + t * pitch[1] + h * pitch[2] + d for r in range(R) for t in range(T) for h in range(H) for d in range(D)]
    return len(set(at)) < len(at)


def test_results_that_lie_on_each_other_are_refused():
    """Several workgroups would write the same place.  16 values a head, rows 2 * 3, any order of the three pitches and any distance."""
    import itertools
    kw = dict(head_dim=16, n_heads=1)
    seen = {False: 0, True: 0}
    for T, H in ((1, 1), (1, 3), (2, 1), (3, 2), (4, 3)):
        n = binding.attention_workspace_bytes(_cache(**kw), binding.attention_params(T, H, 1.0))
        for pitch in itertools.product((0, 8, 15, 16, 17, 32, 33, 48, 64, 96, 112, 200, 1000, 1 << 40, (1 << 62) + 5), repeat=3):
            overlap = _places(6, T, H, 16, pitch)
            seen[overlap] += 1
            assert _attention(T=T, q_heads=H, out_pitch=pitch, bytes=n - 1, **kw) == (INVALID if overlap else SMALL), (T, H, pitch)
    assert min(seen.values()) > 1000
    # many heads, tokens and rows
    for T, H, S, B in ((1000, 64, 4, 2), (1 << 13, 8, 1, 256), (1, 32, 1 << 10, 256)):
        row, token, head = side_by_side(T, H, 64)
        many = dict(T=T, q_heads=H, S=S, B=B, bytes=0)
        assert _attention(out_pitch=(row, token, head), **many) == SMALL
        assert _attention(out_pitch=(64, 64 * S * B * H, 64 * S * B), **many) == SMALL      # heads of all rows together
        assert _attention(out_pitch=(row - 1, token, head), **many) == INVALID
        assert _attention(out_pitch=(row, token, head - 1), **many) == INVALID
        assert _attention(out_pitch=(row + 1, token + 1, head), **many) == (SMALL if T == 1 else INVALID)
