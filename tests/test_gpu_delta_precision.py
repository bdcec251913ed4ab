"""What lsh_delta_rule holds between its inputs and its results has 32 bits, whatever their type.

A row's tokens ask for what they themselves wrote: q = k, of length 1 exactly (entries of 0 and +-2^-m), beta 1, no decay.  So a result is the token's value, made
of q's product with the state before the chunk and of what the chunk's tokens wrote, which take each other away: with values of 2^-12 and states of 1 what
is lost of either shows, also behind a rounding to 16 bits.

Tolerance, for the root of the mean square.  A sum of n terms of random sign whose squares add up to a^2 rounds n times, each time by 2^-24 of what has been added up
at most, a in the mean: 2^-24 sqrt(n) a.  A result is the sum over the keys' entries (twice: in u, and its own) and over a chunk's tokens three times (T, A U, the
state), so n = 2 k_dim + 192.  What a token's u is off by lies in the state along its key, of length 1; later tokens turn that by maps that make nothing longer, and a
result sees it through a key: not more than u was off.  There are up to 64 of these in a chunk, each seen with a weight of 1 / sqrt(entries) >= 1 / 16 in the mean,
some 1 to 2 times a result's own altogether; 4 times is allowed.  a is 1 for random signs; for entries and states of one sign sums grow to
sqrt(entries) times the states' mean, 0.8.  On top comes the rounding of the result."""
import numpy as np
import pytest

from test_gpu_packed import TYPES, half_step, in_64, on_gpu, torch_type, workspace

pytestmark = pytest.mark.gpu


def rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("one_sign", [False, True])
@pytest.mark.parametrize("R,H,T,Dk,entries,Dv", [(1, 2, 64, 64, 64, 32), (2, 3, 64, 32, 16, 16), (1, 1, 200, 256, 256, 48), (2, 1, 100, 96, 64, 80), (1, 4, 70, 128, 64, 128),
                                                 (40, 20, 64, 64, 64, 32), (30, 10, 70, 192, 64, 48)])
def test_a_value_that_takes_the_states_place(R, H, T, Dk, entries, Dv, one_sign, dtype):
    """(The last two: more than 512 workgroups of 16 columns.)"""
    import torch
    from paper_1806_00588_amd import binding
    rng = np.random.default_rng(Dk + T)
    k = np.zeros((R, T, H, Dk))
    sign = np.ones((R, T, H, entries)) if one_sign else rng.choice([-1.0, 1.0], (R, T, H, entries))
    k[..., rng.permutation(Dk)[:entries]] = sign / np.sqrt(entries)
    state = rng.normal(size=(R, H, Dk, Dv))
    v = in_64(on_gpu(rng.normal(size=(R, T, H, Dv)) * 2.0 ** -12, dtype))
    dp = binding.delta_params(R, 1, T, H, H, Dk, Dv, 1.0)
    key, out = on_gpu(k, dtype), torch.zeros(R, T, H, Dv, dtype=torch_type(dtype), device="cuda")
    to, zero = torch.empty(R, H, Dk, Dv, device="cuda"), torch.zeros(R, T, H, device="cuda")
    binding.delta_rule(dp, key, key, on_gpu(v, dtype), zero, zero + 1, on_gpu(np.abs(state) if one_sign else state), to,
                       workspace(binding.delta_workspace_bytes(dp)), out)
    a = 0.8 * np.sqrt(entries) if one_sign else 1.0
    off, most = rms(in_64(out) - v), 4 * 2.0 ** -24 * np.sqrt(2 * Dk + 192) * a + rms(half_step(v, dtype))
    assert off <= most, (off, most)
