"""Runs token operators against tests/launch_lanes.c and prints what they would launch (a program of its own: it must not share a
process with torch, which loads the real runtime).

argv: the recorder, the library.  stdin: a JSON list of [entry point, arguments]; stdout: a JSON list of {"rc", "launches": [{"kernel",
"lanes", "grid"}, ...]}.  Addresses are numbers that nothing reads: "p" in the arguments, "ws" for a workspace and its bytes.
"""
import ctypes as C
import json
import sys

ADDRESS = 1 << 20


def main():
    recorder = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
    lib = C.CDLL(sys.argv[2])
    recorder.recorder_name.restype = C.c_char_p
    recorder.recorder_lanes.restype = recorder.recorder_grid.restype = C.c_uint64
    out = []
    for name, args in json.load(sys.stdin):
        recorder.recorder_reset()
        values = []
        for a in args:
            if a == "p":
                values.append(C.c_void_p(ADDRESS))
            elif a == "ws":
                values += [C.c_void_p(ADDRESS), C.c_size_t(1 << 50)]
            elif a is None:
                values.append(C.c_void_p(None))
            elif isinstance(a, float):
                values.append(C.c_float(a))
            else:
                values.append(C.c_int64(a))
        rc = getattr(lib, name)(*values)
        out.append({"rc": rc, "launches": [
            {"kernel": recorder.recorder_name(i).decode(), "lanes": [recorder.recorder_lanes(i, d) for d in range(3)],
             "grid": [recorder.recorder_grid(i, d) for d in range(3)]} for i in range(recorder.recorder_count())]})
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    main()
