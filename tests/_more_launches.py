"""What the entry points around the linear layer would launch, without a GPU: calls in a
process of their own, recorded as in ``_launches``."""
from __future__ import annotations

import ctypes
import json
import os
import subprocess
import sys

from _launches import HERE, POINTERS, Rows, _rows


class GroupRows(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("pitch", ctypes.c_int64),
                ("scale_pitch", ctypes.c_int64), ("rows", ctypes.c_int32), ("channels", ctypes.c_int32),
                ("group", ctypes.c_int32), ("scale_dtype", ctypes.c_int32)]


def _call(lib, op: str, m: int, c: int, k: int = 0, bits: int = 4, group: int = 0, scales: int = 1, experts: int = 0,
          dtype: int = 0, residual: bool = False, gain: int = 2) -> int:
    """One call of m rows, c channels and k outputs (of each expert)."""
    i32, i64, vp, f64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_double, ctypes.c_size_t
    P, need, ref = POINTERS, ctypes.c_size_t(0), ctypes.byref
    if op == "norm":
        add = (vp(P[1]), i64(c), vp(P[2]), i64(c)) if residual else (None, i64(0), None, i64(0))
        return lib.qconv_norm_rows(vp(P[0]), i64(c), *add, i32(dtype), vp(P[3]), i32(gain), f64(1e-6), i32(m), i32(c),
                                   vp(P[4]), i64((c + 15) // 16 * 16), vp(P[5]), vp(P[6]), None)
    if op == "norm_grad":
        lib.qconv_norm_rows_grad_workspace_bytes(i32(m), i32(c), ref(need))
        add = (vp(P[2]), i64(c)) if residual else (None, i64(0))
        return lib.qconv_norm_rows_grad(vp(P[0]), i64(c), vp(P[1]), i64(c), *add, i32(dtype), vp(P[3]), i32(gain), vp(P[4]),
                                        i32(m), i32(c), vp(P[5]), i64(c), vp(P[6]), vp(P[7]), need, None)
    rows = k * max(experts, 1)
    if group:
        w = GroupRows(P[2], P[3], (c // 2 + 15) // 16 * 16, -(-c // group), rows, c, group, scales)
    else:
        w = _rows(2, rows, c, bits)
    form = "_groups" if group else ""
    dealt = (vp(P[6]), i32(experts)) if experts else ()
    name = f"qconv_linear{'_experts' if experts else ''}{form}"
    if op == "forward":
        return getattr(lib, name)(ref(_rows(0, m, c)), ref(w), *dealt, vp(P[8]), i32(dtype), i64(k), None)
    if op == "grad_weight":
        return lib.qconv_linear_experts_grad_weight(vp(P[4]), i32(dtype), i64(k), i32(k), ref(_rows(0, m, c)), *dealt,
                                                    vp(P[8]), i64(c), None)
    scratch = ()
    if not experts:
        lib.qconv_linear_grad_workspace_bytes(i32(m), i32(c), i32(k), ref(need))
        scratch = (vp(P[9]), need)
    return getattr(lib, name + "_grad_input")(vp(P[4]), i32(dtype), i64(k), i32(m), ref(w), *dealt, vp(P[8]), i64(c), *scratch,
                                              None)


def record(tmp, steps: list) -> dict:
    """As ``_launches.record``, for these calls."""
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
