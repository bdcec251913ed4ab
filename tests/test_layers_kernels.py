"""Which kernel a product takes, by the symbols that are launched: no GPU, nothing is run."""
import json
import os
import re
import subprocess
import sys

import pytest

import test_gpu_delta_kernels as delta
import test_gpu_packed_kernels as narrow
import test_gpu_packed_wide as wide

HERE = os.path.dirname(os.path.abspath(__file__))
TYPE = {"f32": 0, "bf16": 1, "f16": 2}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    from test_library_exports import _lib
    _lib()                       # (built, if it was not)
    so = str(tmp_path_factory.mktemp("recorder") / "recorder.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "kernel_recorder.cpp"), "-ldl"])

    def run(calls):
        """For each call (name, arguments) [(kernel, template arguments)]."""
        done = subprocess.run([sys.executable, os.path.join(HERE, "recorded_layer_kernels.py"), so], input=json.dumps(calls), capture_output=True, text=True)
        assert done.returncode == 0, (done.returncode, done.stderr[-2000:])
        out = []
        for (status, names), call in zip(json.loads(done.stdout), calls):
            assert status == 0 and names, call
            out.append([(re.search(r"k_[a-z_]+", n)[0].rstrip("I"), tuple(int(x) for x in re.findall(r"L[ib](\d+)E", n))) for n in names])
        return out
    return run


def product(name, M, N, K, group, dtype, zeros):
    """zeros: of each matrix."""
    kw = dict(N=N, K=K, group=group, M=M, x_type=TYPE[dtype], x_ld=K, out_ld=N)
    of = [dict(zeros=1 << 20) if z else {} for z in zeros]
    return name, dict(kw, gate=of[0], up=of[1]) if name == "gated" else dict(kw, **of[0])


def test_the_wide_cases_take_every_kernel_of_128_rows(kernels):
    """k_packed_tiles<type, row tiles, tiles of outputs, times 32 inputs of a group, gated, 64 rows, zeros of 8>."""
    calls = [product("linear", *case, (z,)) for case in wide.flat(wide.LINEAR) for z in (0, 1)]
    calls += [product("gated", *case, z) for case in wide.flat(wide.GATED) for z in ((0, 0), (1, 1), (1, 0), (0, 1))]
    taken = set()
    for call, launched in zip(calls, kernels(calls)):
        tiles = [args for name, args in launched if name == "k_packed_tiles"]
        assert len(tiles) == 1 and tiles[0][5] == 0, (call, launched)
        taken.add(tiles[0])
    want = {(t, 4, ns, per, gated, 0, eight) for t in (0, 1, 2) for ns in (2, 4) for per in (1, 2, 4) for gated in (0, 1) for eight in (0, 1)
            if not (ns == 4 and per == 1) and not (t == 2 and eight)}       # (no four tiles of groups of 32, and one conversion for fp16)
    assert taken == want, (want - taken, taken - want)


def built(kernel):
    """Template arguments of every kernel of that name in the library."""
    from paper_1806_00588_amd import library_path
    symbols = subprocess.check_output(["nm", "-D", "--defined-only", library_path()], text=True).split()
    return {tuple(int(x) for x in re.findall(r"L[ib](\d+)E", s)) for s in symbols if re.match(r"_ZN7lshbeam\d+%sI" % kernel, s)}


def test_the_cases_take_every_kernel_of_products(kernels):
    every = [(lists.LINEAR, lists.GATED) for lists in (wide, narrow)]
    calls = [product("linear", *case, (z,)) for linear, _ in every for case in wide.flat(linear) for z in (0, 1)]
    calls += [product("gated", *case, z) for _, gated in every for case in wide.flat(gated) for z in ((0, 0), (1, 0))]
    taken = {kernel for launched in kernels(calls) for kernel in launched}
    for name in ("k_packed_rows", "k_packed_tiles", "k_packed_lay"):
        left_out = built(name) - {args for kernel, args in taken if kernel == name}
        assert built(name) and not left_out, (name, left_out)


def test_the_cases_take_every_kernel_of_the_delta_rule(kernels):
    calls = []
    for S, H, Hk, T, Dk, Dv in delta.FEW + delta.CHUNKS + delta.MANY:
        for ty in (0, 1, 2):
            calls.append(("delta", dict(S=S, B=1, T=T, n_heads=H, n_k_heads=Hk, k_dim=Dk, v_dim=Dv, q_type=ty, k_type=ty, v_type=ty, out_type=ty, q_head=Dk,
                                        out_pitch=(T * H * Dv, H * Dv, Dv))))
    taken = {kernel for launched in kernels(calls) for kernel in launched}
    for name in ("k_delta_tokens", "k_delta_prepare", "k_delta_chain", "k_delta_apart"):
        left_out = built(name) - {args for kernel, args in taken if kernel == name}
        assert built(name) and not left_out, (name, left_out)


@pytest.mark.parametrize("name,M,N,K,dtype,kernel", [("linear", 17, 40000, 1000, "f32", "k_packed_rows"), ("linear", 32, 40000, 1000, "f32", "k_packed_rows"),
                                                     ("gated", 24, 16384, 4096, "f32", "k_packed_rows"), ("linear", 64, 40000, 1000, "bf16", "k_packed_rows"),
                                                     ("linear", 40, 40000, 1000, "f32", "k_packed_tiles"), ("gated", 40, 16384, 4096, "bf16", "k_packed_tiles"),
                                                     ("linear", 28, 1000, 16384, "bf16", "k_packed_tiles"), ("linear", 129, 64, 64, "f16", "k_packed_tiles")])
def test_a_product_takes_the_quicker_kernel(kernels, name, M, N, K, dtype, kernel):
    """As both were measured (takes_tiles in lshlayers.hip has the times)."""
    launched, = kernels([product(name, M, N, K, 128, dtype, (0, 0))])
    assert kernel in [k for k, _ in launched]
