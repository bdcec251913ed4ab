"""Run as a program: python recorded_layer_kernels.py LIBRARY, a list of calls as JSON on stdin, [status, kernels' symbols] of each as JSON on stdout.
LIBRARY is kernel_recorder.cpp, built.  A process of its own, because the recorder stands in front of the HIP runtime in it."""
import ctypes
import json
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))


def main():
    recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    recorder.recorder_name.restype = ctypes.c_char_p
    sys.path[:0] = [os.path.dirname(HERE), HERE]
    import test_layers_refusals as calls       # (argument lists with made-up addresses)
    out = []
    for name, kw in json.load(sys.stdin):
        recorder.recorder_begin(-1)
        recorder.recorder_names_begin()
        status = {"linear": calls._linear, "gated": calls._gated, "delta": calls._delta}[name](**kw)
        out.append((status, [recorder.recorder_name(i).decode() for i in range(recorder.recorder_count())]))
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    main()
