"""Run as a program: python recorded_launches.py LIBRARY, a list of calls as JSON on stdin, what each would launch as JSON on stdout.
LIBRARY is launch_recorder.cpp, built.  A process of its own, because the recorder stands in front of the HIP runtime in it."""
import ctypes
import json
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))


def main():
    recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    sys.path[:0] = [os.path.dirname(HERE), HERE]
    import test_decoder_refusals as calls      # (argument lists with made-up addresses)
    out = []
    for name, refuse, kw in json.load(sys.stdin):
        recorder.recorder_begin(refuse)
        status = {"attention": calls._attention, "select": calls._select, "advance": calls._advance, "write": calls._write}[name](**kw)
        launches = []
        for i in range(recorder.recorder_count()):
            at = (ctypes.c_uint64 * 3)()
            recorder.recorder_get(i, at)
            launches.append(list(at))
        out.append({"status": status, "launches": launches, "last_error": recorder.hipGetLastError()})
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    main()
