"""Pins of the references in oracle/decoder.py against torch's own functions on the CPU."""
import numpy as np
import torch

from oracle import decoder


def test_e4m3_is_torchs():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(np.nan_to_num(every, nan=-1.0), np.nan_to_num(decoder.E4M3, nan=-1.0))
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 0.02, every[np.isfinite(every)],
                        (decoder.E4M3[:126] + decoder.E4M3[1:127]) / 2]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(decoder.to_e4m3(x), want)
    assert list(decoder.to_e4m3(np.array([np.nan, np.inf, -np.inf])) & 127) == [127] * 3


def test_selection_is_log_softmax_and_topk():
    rng = np.random.default_rng(1)
    x, bs = rng.standard_normal((6, 50)), rng.standard_normal(6)
    beam, word, score, lse, _ = decoder.select(x, bs, 2, 3, 5)
    lp = torch.log_softmax(torch.from_numpy(x), 1) + torch.from_numpy(bs)[:, None]
    v, i = lp.view(2, 150).topk(5)
    assert np.allclose(score, v.numpy(), rtol=0, atol=1e-12) and np.array_equal(beam * 50 + word, i.numpy())
    assert np.allclose(lse, torch.logsumexp(torch.from_numpy(x), 1).numpy(), rtol=0, atol=1e-12)


def test_attention_is_softmax_of_products():
    rng = np.random.default_rng(2)
    codes = rng.integers(0, 120, (2, 5, 2, 16, 32)).astype(np.uint8)
    pool = decoder.Pool(codes[0], codes[1], np.full((5, 2), 0.01), np.full((5, 2), 0.5))
    q = rng.standard_normal((1, 3, 4, 32))
    out, lse, _, _ = decoder.attention(pool, q, np.array([[4, 1, 0]]), [37], 0.3)
    k = np.concatenate([decoder.E4M3[codes[0][i]] * 0.01 for i in (4, 1, 0)], axis=1)[:, :37]
    v = np.concatenate([decoder.E4M3[codes[1][i]] * 0.5 for i in (4, 1, 0)], axis=1)[:, :37]
    for t in range(3):
        for h in range(4):
            s = torch.from_numpy(k[h // 2][:35 + t] @ q[0, t, h]) * 0.3
            assert np.allclose(out[0, t, h], torch.softmax(s, 0).numpy() @ v[h // 2][:35 + t]) and np.isclose(lse[0, t, h], torch.logsumexp(s, 0))


def test_layout_there_and_back():
    rng = np.random.default_rng(3)
    codes = rng.integers(0, 256, (2, 3, 2, 32, 48)).astype(np.uint8)
    pool = decoder.Pool(codes[0], codes[1], np.ones((3, 2)), np.ones((3, 2)))
    k, v = pool.layout()
    assert k.shape == (3, 2, 3, 32, 16) and v.shape == (3, 2, 2, 48, 16)
    assert k[1, 0, 2, 5, 7] == codes[0][1, 0, 5, 39] and v[2, 1, 1, 40, 3] == codes[1][2, 1, 19, 40]
    back = decoder.Pool.from_layout(k, v, pool.k_scale, pool.v_scale)
    assert np.array_equal(back.k, pool.k) and np.array_equal(back.v, pool.v)
