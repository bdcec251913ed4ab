"""Rows times weights of 4 bits, every kernel that is built: sizes whose plans take them (test_layers_kernels.py says that none is left out), of every type, group and with
and without zeros.  Tolerances and checks as in test_gpu_packed_wide.py."""
import numpy as np
import pytest

import test_gpu_packed_wide as wide
from test_gpu_packed import TYPES, check_quantize

pytestmark = pytest.mark.gpu

EVERY = [(t, g) for t in TYPES for g in (32, 64, 128)]
# up to 16 rows, 8 and 16 waves, a tile and two tiles a wave; up to 32; 64 rows a workgroup, a tile and two
LINEAR = [(M, N, K, EVERY) for M, N, K in ((3, 300, 500), (12, 2100, 2100), (13, 4509, 520), (11, 8201, 520), (30, 300, 300), (40, 4500, 300), (130, 200, 520), (2050, 500, 300))]
GATED = [(M, N, K, EVERY) for M, N, K in ((3, 300, 500), (12, 4100, 1100), (30, 300, 300), (130, 200, 520))]


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,N,K,group,dtype", wide.flat(LINEAR))
def test_linear(M, N, K, group, dtype, zeros):
    wide.test_linear(M, N, K, group, dtype, zeros)


@pytest.mark.parametrize("zeros", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("M,N,K,group,dtype", wide.flat(GATED))
def test_gated(M, N, K, group, dtype, zeros):
    wide.test_gated(M, N, K, group, dtype, zeros)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("scale", ["f16", "bf16"])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantize(dtype, scale, zeros, group):
    """(And the values that are read back, in each type.)"""
    rng = np.random.default_rng(group)
    check_quantize(rng.normal(size=(35, 333)) * np.exp(rng.normal(size=(35, 1))), group, dtype, scale, zeros, pitch=2)
