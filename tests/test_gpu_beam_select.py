"""lsh_beam_select against oracle/decoder.py.

How far a result may be off, before its first run: a term of a row's sum errs by an ulp of the exponential and half an ulp for each of
up to three fp32 sums, under 2^-21 of it in all, so lse by under 2^-21 (and its rounding to fp32, 2^-24 of it); a score by the same and its
own rounding.  Pairs are the oracle's, place by place, unless the oracle's scores lie closer than twice 2^-21 there: rows of the same
sentence can change places then, words of one row never."""
import numpy as np
import pytest

import oracle.decoder as plain
from gpu_harness import to_dev

pytestmark = pytest.mark.gpu
LSE = 2.0 ** -21
TYPES = {"f32": "float32", "bf16": "bfloat16", "f16": "float16"}


def run(x, bs, S, B, N, allowed=None, fill=-7, stream=None):
    """One call; x a device tensor [S*B, V], allowed int32 bits.  Returns numpy (beam, word, score, lse)."""
    import torch
    from paper_1806_00588_amd import binding
    sp = binding.select_params(S, B, x.shape[1], N)
    ws = torch.full((binding.select_workspace_bytes(sp),), 255, dtype=torch.uint8, device="cuda")
    ob, ow = (torch.full((S, N), fill, dtype=torch.int32, device="cuda") for _ in range(2))
    osc, lse = torch.full((S, N), 123.0, device="cuda"), torch.full((S * B,), 123.0, device="cuda")
    binding.beam_select(sp, x, bs, ws, ob, ow, osc, allowed=allowed, lse=lse, stream=stream)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in (ob, ow, osc, lse)]


def bits_of(allowed):
    """int32 bits of truth values [rows, V]."""
    rows, V = allowed.shape
    padded = np.zeros((rows, (V + 31) // 32 * 32), dtype=bool)
    padded[:, :V] = allowed
    return np.packbits(padded, axis=1, bitorder="little").view(np.int32)


def check(got, x, bs, S, B, N, allowed=None):
    gb, gw, gs, gl = got
    ob, ow, osc, lse, every = plain.select(x, bs, S, B, N, allowed)
    good = np.isfinite(lse)
    assert np.array_equal(gl[~good], lse[~good].astype(np.float32), equal_nan=True)
    assert np.all(np.abs(gl[good] - lse[good]) <= LSE + 2.0 ** -24 * np.abs(lse[good]))
    got_any = ob >= 0
    assert np.array_equal(gb >= 0, got_any) and np.all(gw[~got_any] == -1) and np.all(gb[~got_any] == -1) and np.all(np.isneginf(gs[~got_any]))
    for s in range(S):
        n = int(got_any[s].sum())
        pairs = list(zip(gb[s, :n].tolist(), gw[s, :n].tolist()))
        assert len(set(pairs)) == n
        for i, (b, w) in enumerate(pairs):
            mine = every[s, b, w]
            assert abs(gs[s, i] - mine) <= LSE + 2.0 ** -24 * abs(mine), (s, i, b, w, gs[s, i], mine)
            if (b, w) != (ob[s, i], ow[s, i]):
                assert abs(mine - osc[s, i]) <= 2 * LSE, (s, i, (b, w), (ob[s, i], ow[s, i]), mine, osc[s, i])
                assert any(b != p[0] for p in zip(ob[s, :n].tolist(), ow[s, :n].tolist()))
        assert np.all(np.diff(gs[s, :n]) <= 0)


def inputs(seed, S, B, V, dtype, spread=2.5):
    import torch
    rng = np.random.default_rng(seed)
    x = torch.from_numpy((rng.standard_normal((S * B, V)) * spread).astype(np.float32)).to(getattr(torch, TYPES[dtype]))
    bs = (-8 + rng.standard_normal(S * B)).astype(np.float32)
    return rng, x, bs


# small: one launch up to 64 pieces of 512 words a sentence; above: two
SHAPES = [(1, 1, 1, 1), (1, 1, 1, 5), (1, 4, 7, 4), (2, 3, 511, 3), (1, 3, 512, 40), (3, 2, 513, 256), (1, 4, 1000, 4), (1, 12, 2560, 12),
          (1, 64, 512, 64), (1, 65, 512, 65), (1, 1, 32768, 7), (1, 1, 32769, 256), (2, 17, 4099, 34), (1, 5, 40000, 5), (3, 12, 12001, 9),
          (1, 256, 130, 256), (1, 256, 1111, 200), (1, 2, 200003, 10), (70, 3, 3001, 3)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("S,B,V,N", SHAPES)
def test_matches_plain(S, B, V, N, dtype):
    _, x, bs = inputs(V + B, S, B, V, dtype)
    check(run(x.cuda(), to_dev(bs), S, B, N), x.double().numpy(), bs, S, B, N)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("S,B,V,N", [(2, 3, 511, 3), (1, 5, 40001, 7), (4, 17, 3001, 20)])
def test_rows_of_any_pitch_and_start(S, B, V, N, dtype):
    import torch
    _, x, bs = inputs(5, S, B, V, dtype)
    for pitch, start in ((V + 1, 1), (V + 13, 3), (V + 64, 0)):
        wide = torch.full((S * B, pitch + start), 50.0, dtype=x.dtype, device="cuda")[:, start:]
        wide[:, :V] = x.cuda()
        check(run(wide[:, :V], to_dev(bs), S, B, N), x.double().numpy(), bs, S, B, N)


@pytest.mark.parametrize("V", [33, 1000, 3001, 40000])
@pytest.mark.parametrize("one_row", [False, True])
def test_allowed_words(V, one_row):
    import torch
    S, B, N = 3, 5, 8
    rng, x, bs = inputs(V, S, B, V, "f32")
    allowed = rng.random((1 if one_row else S * B, V)) < 0.1
    if not one_row:
        allowed[4] = False                             # a beam that nothing may follow
        allowed[5:10] = False                          # a sentence with two words in all
        allowed[6, V - 1] = allowed[8, 0] = True
    every = np.broadcast_to(allowed, (S * B, V))
    y = x.numpy().copy()
    y[~every] = rng.choice([np.nan, np.inf, -np.inf, np.finfo(np.float32).min, 1e30], int((~every).sum()))   # what stands there does not count
    wide = torch.full((allowed.shape[0], (V + 31) // 32 + 2), -1, dtype=torch.int32, device="cuda")
    wide[:, :(V + 31) // 32] = torch.from_numpy(bits_of(allowed)).cuda()
    for bits in (to_dev(bits_of(allowed)), wide):
        check(run(to_dev(y), to_dev(bs), S, B, N, allowed=bits), x.double().numpy(), bs, S, B, N, every)


@pytest.mark.parametrize("V", [700, 5000, 70000])
def test_extreme_values(V):
    S, B, N = 2, 6, 10
    low = np.finfo(np.float32).min
    rng, x, bs = inputs(V + 1, S, B, V, "f32")
    x = x.numpy()
    x[0, :] = low                                      # nothing but the lowest value: as likely as each other
    x[1, 3:] = -np.inf                                 # three words
    x[2, :] = -np.inf                                  # none
    x[3, V // 2] = np.nan
    x[4, V - 1] = np.inf
    x[5, ::2] = low                                    # every other word masked
    x[6] += 3e38                                       # sums of huge ones
    x[7, :] = 0.0
    bs[8] = -np.inf                                    # a dead beam
    bs[9] = np.nan
    bs[10] = np.inf
    check(run(to_dev(x), to_dev(bs), S, B, N), x.astype(np.float64), bs, S, B, N)


@pytest.mark.parametrize("value", [0.0, -5.5, np.float32(np.finfo(np.float32).min)])
@pytest.mark.parametrize("B,V,N", [(1, 100, 9), (4, 1000, 256), (3, 40000, 100), (2, 33000, 256), (1, 3000, 256)])
def test_ties_go_to_the_lowest_beam_and_word(B, V, N, value):
    x = np.full((B, V), value, dtype=np.float32)
    bs = np.zeros(B, dtype=np.float32)
    gb, gw, gs, _ = run(to_dev(x), to_dev(bs), 1, B, N)
    n = min(N, B * V)
    assert np.array_equal(gb[0, :n], np.arange(n) // V) and np.array_equal(gw[0, :n], np.arange(n) % V)
    assert np.all(gb[0, n:] == -1)


@pytest.mark.parametrize("B,V,N", [(3, 900, 20), (4, 30000, 50), (1, 5000, 256)])
def test_scores_far_apart_and_huge(B, V, N):
    """The N-th best hundreds behind the best; beam scores of thousands and millions, some beams far behind the others."""
    rng = np.random.default_rng(V)
    x = (rng.standard_normal((2 * B, V)) * 300).astype(np.float32)
    for low in (0.0, -30000.0, -40000.0, -3e6, -1e30):
        bs = (low * (1 + 1e-3 * rng.random(2 * B)) - rng.random(2 * B)).astype(np.float32)
        check(run(to_dev(x), to_dev(bs), 2, B, N), x.astype(np.float64), bs, 2, B, N)
    bs = np.float32([0.0, -20.0, -4000.0, -1e7] * B)[:2 * B]
    y = (rng.standard_normal((2 * B, V)) * 0.01).astype(np.float32)
    check(run(to_dev(y), to_dev(bs), 2, B, N), y.astype(np.float64), bs, 2, B, N)


def test_few_distinct_values():
    """Logits of eight values: thousands of words share a score, and where the N-th best lies many have to be left out."""
    rng = np.random.default_rng(3)
    S, B, V, N = 3, 7, 30011, 200
    x = (rng.integers(0, 8, (S * B, V)) * 0.5).astype(np.float32)
    x[1::2] = x[::2][:x[1::2].shape[0]]                # beams with the same logits, in another sentence too
    bs = np.repeat(np.float32([0.0, 0.0, -3.0]), B)
    bs[14:] = 0.25
    check(run(to_dev(x), to_dev(bs), S, B, N), x.astype(np.float64), bs, S, B, N)


def test_same_bits_every_time_whatever_the_workspace_held():
    import torch
    _, x, bs = inputs(9, 4, 12, 40000, "bf16")
    a = run(x.cuda(), to_dev(bs), 4, 12, 12)
    for _ in range(3):
        b = run(x.cuda(), to_dev(bs), 4, 12, 12, fill=3)
        assert all(np.array_equal(p, q) for p, q in zip(a, b))
    # and rows do not depend on what else is in the call
    torch.cuda.synchronize()
    one = run(x[12:24].cuda(), to_dev(bs[12:24]), 1, 12, 12)
    assert all(np.array_equal(q.reshape(-1), p.reshape(4, 12)[1]) for p, q in zip(a, one))


def test_streams_and_graphs():
    import torch
    from paper_1806_00588_amd import binding
    S, B, V = 2, 6, 50001
    _, x, bs = inputs(11, S, B, V, "f16")
    want = run(x.cuda(), to_dev(bs), S, B, B)
    side = torch.cuda.Stream()
    xd, bd = x.cuda(), to_dev(bs)
    torch.cuda.synchronize()
    got = run(xd, bd, S, B, B, stream=side)
    assert all(np.array_equal(p, q) for p, q in zip(want, got))
    sp = binding.select_params(S, B, V)
    ws = torch.empty(binding.select_workspace_bytes(sp), dtype=torch.uint8, device="cuda")
    ob, ow = (torch.empty((S, B), dtype=torch.int32, device="cuda") for _ in range(2))
    osc = torch.empty((S, B), device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.beam_select(sp, xd, bd, ws, ob, ow, osc)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.beam_select(sp, xd, bd, ws, ob, ow, osc)
    for k in range(3):
        ob.fill_(-9), osc.fill_(7.0), ws.fill_(k)
        if k == 2:
            xd.mul_(-1.0)
            want = run(xd, bd, S, B, B)
        g.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(p, q.cpu().numpy()) for p, q in zip(want, (ob, ow, osc)))


def test_binding_refuses():
    import torch
    from paper_1806_00588_amd import binding
    S, B, V = 2, 3, 100
    sp = binding.select_params(S, B, V)
    ws = torch.empty(binding.select_workspace_bytes(sp), dtype=torch.uint8, device="cuda")
    x, bs = torch.zeros(6, V, device="cuda"), torch.zeros(6, device="cuda")
    i, f = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, device="cuda")
    ok = dict(logits=x, beam_scores=bs, workspace=ws, out_beam=i, out_word=i.clone(), out_score=f)
    for bad in ({"logits": x.double()}, {"logits": x[:5]}, {"logits": x.t().contiguous().t()}, {"logits": x.cpu()}, {"beam_scores": bs[:5]},
                {"beam_scores": bs.half()}, {"out_beam": i.long()}, {"out_beam": i[:4]}, {"out_score": f[:4]}, {"allowed": i.view(6, 1)},
                {"allowed": torch.zeros(2, 4, dtype=torch.int32, device="cuda")}, {"lse": f[:3]}):
        with pytest.raises(ValueError):
            binding.beam_select(sp, **{**ok, **bad})
    with pytest.raises(binding.LshBeamError) as e:
        binding.beam_select(sp, **{**ok, "workspace": ws[:-256]})
    assert e.value.status == 6


@pytest.mark.parametrize("V", [5000, 20001])
def test_rows_far_apart(V):
    """Offsets that pass 32 bits: a pitch of more than 2^29 words."""
    import torch
    S, B, pitch = 2, 4, (1 << 29) + 3
    _, x, bs = inputs(12, S, B, V, "bf16")
    room = torch.empty((S * B - 1) * pitch + V, dtype=torch.bfloat16, device="cuda")
    far = room.as_strided((S * B, V), (pitch, 1))
    far.copy_(x.cuda())
    torch.cuda.synchronize()
    want, got = run(x.cuda(), to_dev(bs), S, B, B), run(far, to_dev(bs), S, B, B)
    assert all(np.array_equal(p, q) for p, q in zip(want, got))


# more than 16384 tiles of 128 words in a sentence, or 256 units of 64 of a row: found by way of the waves' parts
MANY = [(1, 256, 9000, 256), (2, 130, 17001, 34), (1, 20, 150001, 20), (1, 5, 500003, 256)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("S,B,V,N", MANY)
def test_many_tiles(S, B, V, N, dtype):
    _, x, bs = inputs(V, S, B, V, dtype)
    check(run(x.cuda(), to_dev(bs), S, B, N), x.double().numpy(), bs, S, B, N)


@pytest.mark.parametrize("B,V,N", [(40, 120001, 256), (20, 150000, 30), (256, 9000, 3)])
def test_many_tiles_of_ties(B, V, N):
    x = np.full((B, V), 1.5, dtype=np.float32)
    gb, gw, _, _ = run(to_dev(x), to_dev(np.zeros(B, dtype=np.float32)), 1, B, N)
    assert np.all(gb == 0) and np.array_equal(gw[0], np.arange(N))


def test_many_tiles_with_odd_rows_and_masks():
    S, B, V, N = 1, 256, 9000, 40
    rng, x, bs = inputs(21, S, B, V, "f32")
    x = x.numpy()
    x[::7] = np.finfo(np.float32).min
    x[1], x[2, 5], x[3, 6] = -np.inf, np.nan, np.inf
    bs[4:200] = -np.inf
    allowed = rng.random((S * B, V)) < 0.01
    allowed[210] = False
    check(run(to_dev(x), to_dev(bs), S, B, N), x.astype(np.float64), bs, S, B, N)
    check(run(to_dev(x), to_dev(bs), S, B, N, allowed=to_dev(bits_of(allowed))), x.astype(np.float64), bs, S, B, N, allowed)
    y = (rng.standard_normal((B, V)) * 300).astype(np.float32)
    bs = (-3e4 * rng.random(B)).astype(np.float32)
    check(run(to_dev(y), to_dev(bs), S, B, N), y.astype(np.float64), bs, S, B, N)


def test_many_sentences_with_many_results():
    """More than 2^20 results in all."""
    S, B, V, N = 8192, 1, 300, 200
    _, x, bs = inputs(22, S, B, V, "f32")
    check(run(x.cuda(), to_dev(bs), S, B, N), x.double().numpy(), bs, S, B, N)
