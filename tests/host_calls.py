"""The operators' entry points on a machine without a GPU: libtensile.so in a process of its own, where hip_stub.c takes the place of the
HIP runtime.  Every check of the arguments and the choice of kernels run as they do elsewhere; nothing is computed.

    host = Host(folder)                       # builds the stub there
    host("gated_linear", mat(A, 4, 64), ...)  # -> Reply(code, error, launches); the handle and the stream are added

A launch is (the kernel's mangled name, workgroups, threads).  Addresses are numbers that nobody reads."""
from __future__ import annotations

import ctypes
import json
import os
import subprocess
import sys
from collections import namedtuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2105_13336_amd", "libtensile.so")

F32, BF16, F16 = 0, 1, 2                                                # TENSILE_F32, ...
SIZE = {F32: 4, BF16: 2, F16: 2}
Reply = namedtuple("Reply", "code error launches")


def mat(at, rows, cols, ld=None, type=BF16):
    return {"m": [at, rows, cols, cols if ld is None else ld, type]}


def ckpt(q, scale, rows, cols, ld_q=None, ld_scale=None):
    return {"c": [q, scale, rows, cols, cols if ld_q is None else ld_q, (cols + 31) // 32 if ld_scale is None else ld_scale]}


def ptr(at):
    return {"p": at}


class Host:
    def __init__(self, folder):
        if not os.path.exists(LIB):
            from paper_2105_13336_amd.build import build_library
            build_library()
        stub = os.path.join(str(folder), "hip_stub.so")
        subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", "-Wall", os.path.join(HERE, "hip_stub.c"), "-o", stub])
        self.process = subprocess.Popen([sys.executable, os.path.abspath(__file__), stub, LIB], stdin=subprocess.PIPE, stdout=subprocess.PIPE, text=True)

    def __call__(self, name, *args):
        self.process.stdin.write(json.dumps([name, args]) + "\n")
        self.process.stdin.flush()
        return Reply(*json.loads(self.process.stdout.readline()))

    def close(self):
        self.process.stdin.close()
        self.process.wait(30)


def _serve(stub_path, lib_path):
    class Matrix(ctypes.Structure):
        _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("type", ctypes.c_int32)]

    class Ckpt(ctypes.Structure):
        _fields_ = [("q", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld_q", ctypes.c_int64),
                    ("ld_scale", ctypes.c_int64)]

    def given(a):
        if a is None:
            return ctypes.c_void_p(None)
        if isinstance(a, dict):
            (kind, v), = a.items()
            return ctypes.c_void_p(v) if kind == "p" else ctypes.byref(Matrix(*v) if kind == "m" else Ckpt(*v))
        return ctypes.c_double(a) if isinstance(a, float) else ctypes.c_int32(a)

    stub = ctypes.CDLL(stub_path, ctypes.RTLD_GLOBAL)                   # (its symbols come before the runtime's, which the library is linked to)
    lib = ctypes.CDLL(lib_path)
    stub.stub_name.restype = lib.tensile_last_error.restype = ctypes.c_char_p
    ops = ctypes.c_void_p()
    assert lib.tensile_ops_create(ctypes.byref(ops)) == 0
    for line in sys.stdin:
        name, args = json.loads(line)
        stub.stub_forget()
        code = getattr(lib, "tensile_" + name)(ops, *[given(a) for a in args], ctypes.c_void_p(None))
        launches = [(stub.stub_name(k).decode(), stub.stub_grid(k), stub.stub_block(k)) for k in range(stub.stub_launches())]
        print(json.dumps([code, lib.tensile_last_error().decode() if code else "", launches]), flush=True)


if __name__ == "__main__":
    _serve(*sys.argv[1:])
