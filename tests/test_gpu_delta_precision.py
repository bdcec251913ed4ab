"""What lsh_delta_rule holds between its inputs and its results has 32 bits, whatever their type.

A row's tokens ask for what they themselves wrote: keys of length 1 exactly (entries of 0 and +-2^-m), queries some 0.9 times the keys, beta 1, no decay.  So a result
is that factor times the token's value, made of the query's product with the state before the chunk and of what the chunk's tokens wrote, which take each other away: with values
of 2^-12 and states of 1 what is lost of either shows, also behind a rounding to 16 bits.  And the state that is left gives the last key's value for that key.

Tolerance, for the root of the mean square.  A sum of n terms of random sign whose squares add up to a^2 rounds n times, each time evenly over at most half a step of what has been
added up, a sqrt(i / n) in the mean: 2^-24 sqrt(n / 6) a (1 / 3 from the evenness, 1 / 2 from the sum of i / n).  A result is the sum over the keys' entries (twice: in u, and its own) and
over a chunk's tokens three times (T, A U, the state), so n = 2 k_dim + 192.  What a token's u is off by lies in the state along its key, of length 1; later tokens turn that by maps
that make nothing longer, and a result sees it through a key: not more than u was off, and of up to 64 of these, each with a weight of 1 / sqrt(entries) in the mean, once
to twice a result's own altogether; 3 times is allowed.  a is 1 for random signs; for entries and states of one sign sums grow to sqrt(entries) times the states' mean,
0.8.  On top comes the rounding of the result."""
import numpy as np
import pytest

from test_gpu_packed import TYPES, half_step, in_64, on_gpu, torch_type, workspace
from test_gpu_packed_precision import rms

pytestmark = pytest.mark.gpu


def allowed(Dk, entries, one_sign):
    return 3 * 2.0 ** -24 * np.sqrt((2 * Dk + 192) / 6) * (0.8 * np.sqrt(entries) if one_sign else 1.0)


def keys(rng, shape, Dk, entries, one_sign):
    k = np.zeros(shape + (Dk,))
    k[..., rng.permutation(Dk)[:entries]] = (np.ones(shape + (entries,)) if one_sign else rng.choice([-1.0, 1.0], shape + (entries,))) / np.sqrt(entries)
    return k


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("one_sign", [False, True])
@pytest.mark.parametrize("R,H,T,Dk,entries,Dv", [(1, 2, 64, 64, 64, 32), (2, 3, 64, 32, 16, 16), (1, 1, 200, 256, 256, 48), (2, 1, 100, 96, 64, 80), (1, 4, 70, 128, 64, 128),
                                                 (40, 20, 64, 64, 64, 32), (30, 10, 70, 192, 64, 48)])
def test_a_value_that_takes_the_states_place(R, H, T, Dk, entries, Dv, one_sign, dtype):
    """(The last two: more than 512 workgroups of 16 columns.)"""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(Dk + T)
    k = keys(rng, (R, T, H), Dk, entries, one_sign)
    q = in_64(on_gpu(0.9 * k, dtype))
    state = rng.normal(size=(R, H, Dk, Dv))
    v = in_64(on_gpu(rng.normal(size=(R, T, H, Dv)) * 2.0 ** -12, dtype))
    dp = binding.delta_params(R, 1, T, H, H, Dk, Dv, 1.0)
    out = torch.zeros(R, T, H, Dv, dtype=torch_type(dtype), device="cuda")
    to, zero = torch.empty(R, H, Dk, Dv, device="cuda"), torch.zeros(R, T, H, device="cuda")
    binding.delta_rule(dp, on_gpu(q, dtype), on_gpu(k, dtype), on_gpu(v, dtype), zero, zero + 1, on_gpu(np.abs(state) if one_sign else state), to,
                       workspace(binding.delta_workspace_bytes(dp)), out)
    most, want = allowed(Dk, entries, one_sign), v * np.abs(q).max() * np.sqrt(entries)
    off = rms(in_64(out) - want)
    assert off <= most + rms(half_step(want, dtype)), (off, most)
    off = rms((k[:, -1, :, :, None] * in_64(to)).sum(2) - v[:, -1])
    assert off <= most, (off, most)
