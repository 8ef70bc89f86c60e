"""Runs optimizer steps against tests/launch_lanes.c and prints what they would launch (a program of its own: it must not share a process
with torch, which loads the real runtime).

argv: the recorder, the library.  stdin: a JSON list of [elements of every tensor, bits]; stdout: a JSON list of {"rc", "launches"}.
"""
import ctypes as C
import json
import sys

ADDRESS = 1 << 20


class Item(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("scales", C.c_void_p), ("copy", C.c_void_p),
                ("n", C.c_int64), ("scales_stride", C.c_int64), ("weight_decay", C.c_float)]


class Options(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("grad_scale", C.c_double), ("step", C.c_int64),
                ("seed", C.c_uint64), ("lr_device", C.c_void_p), ("grad_scale_device", C.c_void_p), ("step_device", C.c_void_p)]


def main():
    recorder = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
    lib = C.CDLL(sys.argv[2])
    recorder.recorder_name.restype = C.c_char_p
    recorder.recorder_lanes.restype = recorder.recorder_grid.restype = C.c_uint64
    out = []
    for sizes, bits in json.load(sys.stdin):
        recorder.recorder_reset()
        items = (Item * len(sizes))()
        for it, n in zip(items, sizes):
            it.param = it.grad = it.m = it.v = it.scales = it.copy = ADDRESS
            it.n, it.scales_stride = n, -(-n // 128)
        o = Options(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, 0, None, None, None)
        rc = lib.bsr_adamw_batched(items, len(sizes), 1, 1, 1 if bits == 8 else 0, C.byref(o), None)
        out.append({"rc": rc, "launches": [{"kernel": recorder.recorder_name(i).decode(), "lanes": recorder.recorder_lanes(i, 0)}
                                           for i in range(recorder.recorder_count())]})
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    main()
