"""The references of a decoder's layers against hand-made cases."""
import numpy as np

from oracle import layers


def test_places_of_codes():
    assert layers.place(0, 0, 1) == (0, False) and layers.place(0, 4, 1) == (0, True) and layers.place(0, 3, 1) == (3, False)
    assert layers.place(0, 32, 1) == (4, False)                     # the next word of the same lane
    assert layers.place(1, 0, 1) == (16, False)                     # the next output
    assert layers.place(0, 8, 1) == (256, False)                    # the next eight inputs
    assert layers.place(16, 128, 2) == (3 * 1024, False)            # the next tile and part
    codes = np.random.default_rng(0).integers(0, 16, (33, 150))
    assert (layers.unpack(layers.pack(codes), 33, 150) == codes).all()
    g = np.arange(33 * 5).reshape(33, 5)
    assert (layers.to_groups(layers.of_groups(g, (3, 2, 16, 4)), 33, 5) == g).all()


def test_quantize_small():
    half = lambda x: np.float16(x)
    w = np.array([[7.0, -7.0, 3.5, 0.5, 1.5, -0.5]], dtype=np.float32)
    codes, s, z = layers.quantize(w, 32, half, False)
    assert s[0, 0] == 1 and codes.tolist() == [[15, 1, 12, 8, 10, 8]]            # halves to even
    codes, s, z = layers.quantize(np.array([[-1.0, 14.0, 6.5]], dtype=np.float32), 32, half, True)
    assert s[0, 0] == 1 and z[0, 0] == 1 and codes.tolist() == [[0, 15, 7]]
    assert (layers.values(codes, s, z, 32) == [[-1, 14, 6]]).all()
    codes, s, z = layers.quantize(np.zeros((1, 3), dtype=np.float32), 32, half, False)
    assert s[0, 0] == 0 and codes.tolist() == [[8, 8, 8]]


def test_delta_rule_forgets_what_a_key_held():
    """beta 1, no decay, a unit key: afterwards the state gives the new value for that key, and others keep theirs."""
    k = np.eye(4)[None, :, None]                                     # four tokens, four keys
    v = np.arange(12.0).reshape(1, 4, 1, 3)
    zero = np.zeros((1, 4, 1))
    out, S, _ = layers.delta_rule(k, k, v, zero, zero + 1, np.full((1, 1, 4, 3), 9.0), 1.0)
    assert (S[0, 0] == v[0, :, 0]).all() and (out == v).all()
    out, S, _ = layers.delta_rule(k[:, :1], k[:, :1], v[:, :1], zero[:, :1] + np.log(0.5), zero[:, :1], np.full((1, 1, 4, 3), 8.0), 2.0)
    assert np.allclose(S, 4.0) and np.allclose(out, 8.0)
