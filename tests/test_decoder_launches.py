"""What the operators around a decoder would launch, written down by a stand-in for the HIP runtime: no GPU, nothing is run."""
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
LDS = 160 * 1024                 # of a CU
STATIC = 4096                    # more than the attention's kernels have besides what they are launched with


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    from test_library_exports import _lib
    _lib()                       # (built, if it was not)
    so = str(tmp_path_factory.mktemp("recorder") / "recorder.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "launch_recorder.cpp")])

    def run(calls, refuse=-1):
        """[{status, launches [[grid, threads, LDS]], last_error}] of calls (name, arguments)."""
        done = subprocess.run([sys.executable, os.path.join(HERE, "recorded_launches.py"), so], input=json.dumps([(n, refuse, kw) for n, kw in calls]),
                              capture_output=True, text=True)
        assert done.returncode == 0, (done.returncode, done.stderr[-2000:])
        return json.loads(done.stdout)
    return run


def _attention_calls():
    """Every head size and type with every number of rows that a workgroup takes: a row's own, and beams over common blocks."""
    for D in range(16, 257, 16):
        for ty in (0, 1, 2):
            for T in (1, 15, 16, 17, 32, 33, 48, 49, 50, 63, 64, 65, 97, 128, 200, 1000):
                yield dict(head_dim=D, q_type=ty, out_type=ty, T=T, q_heads=2, out_pitch=(2 * T * D, 2 * D, D))
            for B, group in ((4, 1), (12, 4), (16, 1), (17, 1), (12, 3), (25, 2), (5, 10), (8, 8), (64, 1), (13, 5), (256, 16)):
                yield dict(head_dim=D, q_type=ty, out_type=ty, S=1, B=B, q_heads=2 * group, out_pitch=(2 * group * D, 0, D), max_blocks=20000,
                           n_blocks=30000, shared=1 << 20)


def test_every_launch_of_the_attention_has_the_lds_it_asks_for(record):
    calls = list(_attention_calls())
    several = 0
    for kw, got in zip(calls, record([("attention", kw) for kw in calls])):
        assert got["status"] == 0 and got["launches"], (kw, got)
        for grid, threads, lds in got["launches"]:
            assert lds + STATIC <= LDS and threads <= 256 and grid < 1 << 24, (kw, got)
        several += len(got["launches"]) > 1
    assert several > 100         # (calls of more than one launch are among them)


def test_a_launch_that_is_refused_leaves_no_error_behind(record):
    """More LDS than the runtime gives: the call says so, and the caller's next look at HIP's last error finds none."""
    calls = [("attention", dict(T=40, q_heads=2, head_dim=128, out_pitch=(10240, 256, 128))), ("attention", dict(S=1, B=64, q_heads=2, head_dim=128, out_pitch=(256, 0, 128), max_blocks=20000, n_blocks=30000, shared=1 << 20))]
    assert [g["status"] for g in record(calls)] == [0, 0]
    for got in record(calls, refuse=1 << 10):
        assert got["status"] == 5 and got["last_error"] == 0, got
