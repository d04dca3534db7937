"""What the library would launch, without a GPU: its entry points called in a
process of their own in which the HIP runtime's launch functions are recorded
(``launch_recorder.cpp``) and nothing runs.  Pointers are plain integers."""
from __future__ import annotations

import ctypes
import json
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
POINTERS = [i << 40 for i in range(1, 17)]   # far apart, 16-byte aligned


class Rows(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("pitch", ctypes.c_int64),
                ("rows", ctypes.c_int32), ("channels", ctypes.c_int32), ("bits", ctypes.c_int32)]


class Adapters(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("alpha", ctypes.c_void_p), ("row", ctypes.c_void_p),
                ("count", ctypes.c_int32), ("rank", ctypes.c_int32)]


def _rows(at: int, rows: int, channels: int, bits: int = 8) -> Rows:
    return Rows(POINTERS[at], POINTERS[at + 1], (channels * bits // 8 + 15) // 16 * 16, rows, channels, bits)


def _call(lib, op: str, m: int = 0, c: int = 0, k: int = 0, bits: int = 8, dtype: int = 0, adapters: int = 0, rank: int = 0,
          stride: int = 0, dy: int = POINTERS[0], workspace: int = POINTERS[9]) -> int:
    """One call of m rows, c channels and k outputs; stride: the gradient's, 0 for tight rows.
    Operands lie at POINTERS 0 to 7 (rows: codes, then scales), results at POINTERS[8]."""
    i32, i64, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    size, need, P = ctypes.c_size_t, ctypes.c_size_t(0), POINTERS
    dy, workspace = vp(dy), vp(workspace)
    if op == "rows":
        return lib.qconv_quantize_rows(vp(P[0]), i32(dtype), i64(c), i32(m), i32(c), vp(P[1]), i64((c + 15) // 16 * 16),
                                       vp(P[2]), None)
    if op == "linear":
        ad = Adapters(P[4], P[5], P[6], P[7], adapters, rank)
        with_ad = ctypes.byref(ad) if adapters else None
        lib.qconv_linear_workspace_bytes(i32(m), i32(c), with_ad, ctypes.byref(need))
        return lib.qconv_linear(ctypes.byref(_rows(0, m, c)), ctypes.byref(_rows(2, k, c, bits)), with_ad, vp(P[8]),
                                i32(dtype), i64(k), workspace, size(need.value), None)
    sizes = (m, c, k) if op == "grad_input" else (k, c, m)
    lib.qconv_linear_grad_workspace_bytes(*map(i32, sizes), ctypes.byref(need))
    if op == "grad_input":
        return lib.qconv_linear_grad_input(dy, i32(dtype), i64(stride or k), i32(m), ctypes.byref(_rows(2, k, c, bits)),
                                           vp(P[8]), i64(c), workspace, size(need.value), None)
    return lib.qconv_linear_grad_weight(dy, i32(dtype), i64(stride or k), i32(k), ctypes.byref(_rows(2, m, c)),
                                        vp(P[8]), i64(c), workspace, size(need.value), None)


def record(tmp, steps: list) -> dict:
    """The steps in a process of their own.  A step is a call's arguments ({"op": ...}),
    {"device": n} to pretend to be on another device, or {"refuse": n} to refuse the next
    n attributes.  Gives "kernels", the names of all kernels of the library, and
    "events", for each step the pair of its status and what it did: ["launch", device,
    name, "grid", threads, LDS bytes] or ["attribute", device, name, value]."""
    from paper_2202_06819_amd import build
    lib = build.ensure_built()
    stub = os.path.join(str(tmp), "launch_recorder.so")
    if not os.path.exists(stub):
        subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-std=c++17", os.path.join(HERE, "launch_recorder.cpp"), "-o", stub],
                       check=True)
    done = subprocess.run([sys.executable, os.path.abspath(__file__), stub, lib], input=json.dumps(steps), text=True,
                          stdout=subprocess.PIPE, check=True)
    return json.loads(done.stdout)


def _main(stub_path: str, lib_path: str) -> None:
    stub = ctypes.CDLL(stub_path, mode=ctypes.RTLD_GLOBAL)
    lib = ctypes.CDLL(lib_path)
    stub.recorder_event.restype = stub.recorder_kernel.restype = ctypes.c_char_p
    events = []
    for step in json.load(sys.stdin):
        stub.recorder_clear()
        status = 0
        if "device" in step:
            stub.recorder_device(step["device"])
        elif "refuse" in step:
            stub.recorder_refuse(step["refuse"])
        else:
            status = _call(lib, **step)
        events.append([status, [stub.recorder_event(i).decode().split("\t") for i in range(stub.recorder_events())]])
    kernels = [stub.recorder_kernel(i).decode() for i in range(stub.recorder_kernels())]
    json.dump({"kernels": kernels, "events": events}, sys.stdout)


if __name__ == "__main__":
    _main(*sys.argv[1:])
