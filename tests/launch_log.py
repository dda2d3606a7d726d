"""Which kernels the library launches for calls of given sizes, without a
device: a child process loads launch_log.cpp's stand-ins for the HIP runtime
and then the library, and makes the calls with made-up pointers."""
from __future__ import annotations

import ctypes
import json
import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_1910_11971_amd", "libcci.so")
P = 0x10000  # aligned, never dereferenced
ACT = 2


def kernels(calls: list[dict], tmp: str) -> list[list[tuple[str, int, int]]]:
    """Per call its launches in order: kernel, workgroups, threads of one."""
    shim = os.path.join(tmp, "launch_log.so")
    if not os.path.exists(shim):
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", os.path.join(HERE, "launch_log.cpp"), "-o", shim], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), shim], input=json.dumps(calls), capture_output=True,
                       text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    return [[(n, int(g), int(b)) for n, g, b in call] for call in json.loads(r.stdout)]


def _make(lib, c):
    t = 0 if c["dtype"] == "f32" else 1
    i64 = ctypes.c_int64
    p = ctypes.c_void_p(P)
    N, C = i64(c["N"]), i64(c["C"])
    if c["kind"] == "norm":
        return lib.cci_layernorm(p, t, N, C, p, p, ctypes.c_float(1e-5), p, p, p, None)
    if c["kind"] == "norm_bwd":
        return lib.cci_layernorm_bwd(p, p, t, N, C, p, p, p, p, p, p, p, ctypes.c_size_t(1 << 40), None)
    G, K = c["G"], c["K"]
    if c["kind"] == "gated":
        return lib.cci_gated_spmm(p, t, N, C, p, p, i64(c["F"]), G, K, ACT, p, p if c.get("train") else None, None)
    if c["kind"] == "gated_bwd":
        return lib.cci_gated_spmm_bwd(p, p, p, t, N, C, p, p, i64(c["F"]), G, K, ACT, p, p, p, t, None)
    if c["kind"] == "back":
        return lib.cci_spmm_t(p, t, N, i64(c["O"]), p, p, C, G, K, p, 0 if c.get("out") == "f32" else t, None)

    class Adapters(ctypes.Structure):
        _fields_ = [("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("alpha", ctypes.c_void_p), ("rows", ctypes.c_void_p),
                    ("L", ctypes.c_int64), ("R", ctypes.c_int32)]

    a = Adapters(P, P, None, P, c["L"], c["R"])
    return lib.cci_spmm_adapters(p, t, N, C, p, t, p, i64(c["O"]), G, K, ctypes.byref(a), None, p, t, p, ctypes.c_size_t(1 << 50), None)


def _child(shim):
    log = ctypes.CDLL(shim, mode=ctypes.RTLD_GLOBAL)
    log.launch_log_take.restype = ctypes.c_char_p
    lib = ctypes.CDLL(LIB)
    lib.cci_last_error.restype = ctypes.c_char_p
    out = []
    for c in json.load(sys.stdin):
        log.launch_log_take()
        st = _make(lib, c)
        if st != 0:
            raise SystemExit(f"{c}: status {st}: {lib.cci_last_error()}")
        rows = [line.rsplit("|", 2) for line in log.launch_log_take().decode().splitlines()]
        out.append([(re.sub(r"void |cci::|\(anonymous namespace\)::", "", n).split("(")[0].strip(), g, b) for n, g, b in rows])
    print(json.dumps(out))


if __name__ == "__main__":
    _child(sys.argv[1])
