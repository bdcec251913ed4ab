"""What a decoder's layers would launch, written down by a stand-in for the HIP runtime: no GPU, nothing is run."""
import json
import os
import random
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
LDS = 160 * 1024                 # of a CU


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    from test_library_exports import _lib
    _lib()                       # (built, if it was not)
    so = str(tmp_path_factory.mktemp("recorder") / "recorder.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "launch_recorder.cpp")])

    def run(calls, refuse=-1):
        """[{status, launches [[grid, threads, LDS]], last_error}] of calls (name, arguments)."""
        done = subprocess.run([sys.executable, os.path.join(HERE, "recorded_layer_launches.py"), so], input=json.dumps([(n, refuse, kw) for n, kw in calls]),
                              capture_output=True, text=True)
        assert done.returncode == 0, (done.returncode, done.stderr[-2000:])
        return json.loads(done.stdout)
    return run


def products():
    rng = random.Random(1)
    sizes = [1, 16, 64, 100, 1000, 4096, 5001, 16384, 40000, 1 << 20]
    for name in ("linear", "gated"):
        for x_type in (0, 1, 2):
            for group in (32, 64, 128):
                for M in (1, 2, 12, 16, 17, 31, 32, 33, 48, 64, 65, 96, 127, 128, 129, 200, 1000, 4096):
                    for _ in range(4):
                        N, K = rng.choice(sizes), rng.choice(sizes[:-1])
                        yield name, dict(N=N, K=K, M=M, group=group, x_type=x_type, x_ld=1 << 20, out_ld=1 << 24)


def test_every_product_fits_the_chip(record):
    calls = list(products())
    kinds = set()
    for (name, kw), got in zip(calls, record(calls)):
        assert got["status"] == 0 and got["launches"], (kw, got)
        for grid, threads, lds in got["launches"]:
            assert lds < LDS and threads <= 1024 and 0 < grid and grid * threads < 1 << 32, (kw, got)
        kinds.add(tuple(threads for _, threads, _ in got["launches"]))
    # rows with 8 and 16 waves, both with inputs split, many rows, and these with inputs split
    assert kinds == {(512,), (1024,), (512, 256), (1024, 256), (256, 512), (256, 512, 256)}, kinds


def test_every_delta_rule_fits_the_chip(record):
    calls = []
    for k_dim in range(16, 257, 16):
        for ty in (0, 1, 2):
            for T in (1, 2, 12, 13, 20, 21, 64, 65, 5000):
                for S, heads in ((1, 1), (3, 16), (40, 8), (1000, 4)):
                    v_dim = (k_dim * 5 + T) // 16 * 16 % 256 + 16
                    if S * heads * T <= 1 << 22:
                        calls.append(("delta", dict(S=S, B=1, T=T, n_heads=heads, n_k_heads=1, k_dim=k_dim, v_dim=v_dim, q_type=ty, k_type=ty, v_type=ty,
                                                    out_type=ty, out_pitch=(T * heads * v_dim, heads * v_dim, v_dim))))
    chunks = 0
    for (_, kw), got in zip(calls, record(calls)):
        # (pairs of launches, as many as the workspace's turns)
        assert got["status"] == 0 and (len(got["launches"]) == 1 if kw["T"] <= 12 else len(got["launches"]) % 2 == 0 or kw["T"] <= 20), (kw, got)
        for grid, threads, lds in got["launches"]:
            assert lds < LDS and threads in (256, 512) and 0 < grid and grid * threads < 1 << 32, (kw, got)
        chunks += len(got["launches"]) > 1
    assert chunks > 100


def test_a_launch_that_is_refused_leaves_no_error_behind(record):
    """More LDS than the runtime gives: the call says so, and the caller's next look at HIP's last error finds none."""
    calls = [("linear", dict(N=4096, K=4096, M=12, out_ld=4096)), ("gated", dict(N=4096, K=4096, M=200, out_ld=4096)),
             ("delta", dict(T=200, k_dim=256, q_type=0, k_type=0, v_type=0, out_type=0, out_pitch=(200 * 192, 192, 48)))]
    assert [g["status"] for g in record(calls)] == [0, 0, 0]
    for got in record(calls, refuse=1 << 10):
        assert got["status"] == 5 and got["last_error"] == 0, got
