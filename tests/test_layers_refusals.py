"""Calls of a decoder's layers that are refused, through the C ABI and without a GPU: arguments are looked at before anything is launched.
Pointers are made up; none is followed."""
import ctypes

import pytest

from paper_1806_00588_amd import binding
from test_library_exports import _lib

INVALID, UNSUPPORTED, SMALL = 1, 2, 6
P = 1 << 20                        # an address at a multiple of 256
BIG = 1 << 40
PARAMS = dict(N=100, K=300, group=64)
BAD_PARAMS = [{"N": 0}, {"N": -1}, {"N": (1 << 24) + 1}, {"K": 0}, {"K": (1 << 20) + 1}, {"group": 0}, {"group": 16}, {"group": 96}, {"group": 256}]
BAD_WEIGHTS = [{"codes": None}, {"codes": P + 8}, {"scales": None}, {"scales": P + 2}, {"zeros": P + 4}, {"scale_dtype": 0}, {"scale_dtype": 3}]
IDS = lambda k: ",".join("%s=%s" % i for i in k.items())


def _params(kw):
    return binding.PackedParams(*[kw.get(n, PARAMS[n]) for n in ("N", "K", "group")])


def _weights(kw):
    return binding._WeightPointers(kw.get("codes", P), kw.get("scales", P), kw.get("zeros", None), kw.get("scale_dtype", 2))


def _quantize(**kw):
    return _lib().lsh_packed_quantize(ctypes.byref(_params(kw)), kw.get("w", P), ctypes.byref(binding._Matrix(kw.get("dtype", 0), kw.get("ld", 1 << 20))),
                                      ctypes.byref(_weights(kw)), None)


def _values(**kw):
    return _lib().lsh_packed_values(ctypes.byref(_params(kw)), ctypes.byref(_weights(kw)), kw.get("w", P),
                                    ctypes.byref(binding._Matrix(kw.get("dtype", 0), kw.get("ld", 1 << 20))), None)


BAD_MATRIX = [{"w": None}, {"w": P + 2}, {"w": P + 1, "dtype": 1}, {"dtype": 3}, {"dtype": -1}, {"ld": 299}]


@pytest.mark.parametrize("kw", BAD_PARAMS + BAD_WEIGHTS + BAD_MATRIX, ids=IDS)
@pytest.mark.parametrize("call", [_quantize, _values], ids=["quantize", "values"])
def test_quantize_refuses(call, kw):
    assert call(**kw) == INVALID


def test_quantize_of_more_than_a_launch():
    assert _quantize(N=1 << 24, K=1 << 20) == UNSUPPORTED and _values(N=1 << 24, K=1 << 20) == UNSUPPORTED
    assert _lib().lsh_packed_quantize(None, P, ctypes.byref(binding._Matrix(0, 300)), ctypes.byref(_weights({})), None) == INVALID
    assert _lib().lsh_packed_quantize(ctypes.byref(_params({})), P, None, ctypes.byref(_weights({})), None) == INVALID
    assert _lib().lsh_packed_quantize(ctypes.byref(_params({})), P, ctypes.byref(binding._Matrix(0, 300)), None, None) == INVALID


def _linear(**kw):
    x, out = binding._Matrix(kw.get("x_type", 1), kw.get("x_ld", 1 << 20)), binding._Matrix(kw.get("out_type", 0), kw.get("out_ld", 1 << 24))
    return _lib().lsh_packed_linear(ctypes.byref(_params(kw)), ctypes.byref(_weights(kw)), kw.get("M", 5), kw.get("x", P), ctypes.byref(x),
                                    kw.get("bias"), kw.get("add"), kw.get("add_ld", 100), kw.get("ws", P), kw.get("bytes", BIG), kw.get("out", P),
                                    ctypes.byref(out), None)


def _gated(**kw):
    x, out = binding._Matrix(kw.get("x_type", 1), kw.get("x_ld", 1 << 20)), binding._Matrix(kw.get("out_type", 0), kw.get("out_ld", 1 << 24))
    return _lib().lsh_packed_gated(ctypes.byref(_params(kw)), ctypes.byref(_weights(kw.get("gate", kw))), ctypes.byref(_weights(kw.get("up", kw))),
                                   kw.get("M", 5), kw.get("x", P), ctypes.byref(x), kw.get("act", 0), kw.get("ws", P), kw.get("bytes", BIG),
                                   kw.get("out", P), ctypes.byref(out), None)


BAD_ROWS = [{"M": 0}, {"M": -3}, {"M": (1 << 20) + 1}, {"x": None}, {"x": P + 1}, {"x": P + 2, "x_type": 0}, {"x_type": 3}, {"x_ld": 299}, {"out": None},
            {"out": P + 2}, {"out_type": -1}, {"out_ld": 99}, {"ws": None}, {"ws": P + 128}]


@pytest.mark.parametrize("kw", BAD_PARAMS + BAD_WEIGHTS + BAD_ROWS + [{"bias": P + 2}, {"add": P, "add_ld": 99}, {"add": P + 2}], ids=IDS)
def test_linear_refuses(kw):
    assert _linear(**kw) == INVALID


@pytest.mark.parametrize("kw", BAD_PARAMS + BAD_WEIGHTS + BAD_ROWS + [{"act": -1}, {"act": 3}, {"gate": {"scale_dtype": 1}, "up": {"scale_dtype": 2}},
                                                                      {"gate": {}, "up": {"codes": None}}], ids=IDS)
def test_gated_refuses(kw):
    assert _gated(**kw) == INVALID


def test_packed_workspace():
    lib = _lib()
    for M in (1, 40, 300):
        n = binding.packed_workspace_bytes(binding.packed_params(100, 300, 64), M)
        assert n > 0 and _linear(M=M, bytes=n - 1) == SMALL and _gated(M=M, bytes=n - 1) == SMALL
    assert all(lib.lsh_packed_workspace_bytes(ctypes.byref(_params(kw)), 1) == 0 for kw in BAD_PARAMS)
    assert lib.lsh_packed_workspace_bytes(None, 1) == 0 and lib.lsh_packed_workspace_bytes(ctypes.byref(_params({})), 0) == 0


DELTA = dict(S=2, B=3, T=4, n_heads=4, n_k_heads=2, k_dim=64, v_dim=48, scale=0.125)
BAD_DELTAS = [{"S": 0}, {"B": 0}, {"B": 257}, {"S": 1 << 20}, {"T": 0}, {"T": (1 << 20) + 1}, {"n_heads": 0}, {"n_k_heads": 0}, {"n_heads": 5}, {"n_heads": 65536},
              {"k_dim": 0}, {"k_dim": 8}, {"k_dim": 40}, {"k_dim": 272}, {"v_dim": 0}, {"v_dim": 20}, {"v_dim": 272}]


def _delta(**kw):
    p = binding.delta_params(**{k: kw.get(k, v) for k, v in DELTA.items()})
    a = dict(q=P, k=P, v=P, decay=P, beta=P, state_in=P, parents=None, n_new=None, state_out=BIG, ws=P, bytes=BIG, out=P, q_type=1, k_type=1, v_type=1,
             out_type=1, q_head=64, out_pitch=(4 * 4 * 48, 4 * 48, 48))
    a.update({k: v for k, v in kw.items() if k not in DELTA})
    q, k = binding._Rows(a["q_type"], 512, 128, a["q_head"]), binding._Rows(a["k_type"], 512, 128, 64)
    v, out = binding._Rows(a["v_type"], 768, 192, 48), binding._Rows(a["out_type"], *a["out_pitch"])
    return _lib().lsh_delta_rule(ctypes.byref(p), a["q"], ctypes.byref(q), a["k"], ctypes.byref(k), a["v"], ctypes.byref(v), a["decay"], a["beta"],
                                 a["state_in"], a["parents"], a["n_new"], a["state_out"], a["ws"], a["bytes"], a["out"], ctypes.byref(out), None)


@pytest.mark.parametrize("kw", BAD_DELTAS + [
    {"scale": float("inf")}, {"scale": float("nan")}, {"q": None}, {"k": None}, {"v": None}, {"out": None}, {"q": P + 1}, {"k": P + 1}, {"v": P + 1}, {"out": P + 1},
    {"q_type": 0}, {"k_type": 2}, {"v_type": 0}, {"out_type": 0}, {"q_head": -64}, {"decay": None}, {"beta": None}, {"decay": P + 2}, {"state_out": None},
    {"state_out": BIG + 8}, {"state_in": P + 4}, {"parents": P + 2}, {"n_new": P + 1}, {"ws": None}, {"ws": P + 64},
    {"state_out": P, "parents": P}, {"state_out": P + 1024}, {"state_out": P - 1024}, {"out_pitch": (768, 192, 32)}, {"out_pitch": (0, 192, 48)}],
    ids=IDS)
def test_delta_refuses(kw):
    assert _delta(**kw) == INVALID


def test_delta_workspace():
    p = lambda **kw: binding.delta_params(**dict(DELTA, **kw))
    for T in (1, 500):
        n = binding.delta_workspace_bytes(p(T=T))
        assert n > 0 and _delta(T=T, bytes=n - 1, out_pitch=(T * 192, 192, 48)) == SMALL
    assert all(binding.delta_workspace_bytes(p(**kw)) == 0 for kw in BAD_DELTAS)
    assert binding.delta_workspace_bytes(p(S=1 << 12, T=1 << 12)) == 0 and _delta(S=1 << 12, T=1 << 12) == UNSUPPORTED
    assert _lib().lsh_delta_workspace_bytes(None) == 0
