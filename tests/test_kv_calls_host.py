"""The host side of the paged cache (kv_api.cpp) on a stand-in for the HIP runtime: which
device its calls go to and what they hand to the kernels.  No GPU."""

from __future__ import annotations

import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2607_18253_amd.kv import KvConfig, KvPagesArg, KvRowsArg

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2607_18253_amd", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    out = str(tmp_path_factory.mktemp("kv") / "libkvhost.so")
    stub = os.path.join(HERE, "hip_stub")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", stub, os.path.join(CSRC, "kv_api.cpp"),
                    os.path.join(stub, "kv_host.cpp"), "-o", out], check=True)
    L = C.CDLL(out)
    vp, i32 = C.c_void_p, C.c_int32
    L.lar_kv_plan.argtypes = [vp, i32, vp, vp, i32, i32]
    L.lar_kv_append.argtypes = [vp, vp, vp, vp, vp, i32]
    L.lar_kv_read.argtypes = [vp, vp, vp, i32, vp, vp]
    L.lar_kv_attend.argtypes = [vp, vp, vp, vp, i32, C.c_double, vp, vp]
    for f in (L.lar_kv_sync, L.lar_kv_destroy):
        f.argtypes = [vp]
    L.lar_kv_create.argtypes = [C.POINTER(vp), vp]
    L.lar_kv_error_string.argtypes, L.lar_kv_error_string.restype = [vp], C.c_char_p
    return L


class Handle:
    """A handle of 8 and 2 heads of 64, pages and rows that no kernel looks at."""

    def __init__(self, lib, max_seqs=8, max_tokens=256):
        self.L, self.h = lib, C.c_void_p()
        cfg = KvConfig(8, 2, 64, 1, 1, 16, max_seqs, max_tokens, 0, None)
        assert lib.lar_kv_create(C.byref(self.h), C.byref(cfg)) == 0
        self.pages = KvPagesArg(4096, 8192, None, None, 64)
        self.q, self.kv = KvRowsArg(4096, 512, 64), KvRowsArg(4096, 128, 64)

    def plan(self, q_len, ctx, window=0, sinks=0):
        q, c = np.array(q_len, np.int32), np.array(ctx, np.int32)
        return self.L.lar_kv_plan(self.h, len(q), q.ctypes.data, c.ctypes.data, window, sinks)

    def append(self, k=None):
        k = C.byref(self.kv if k is None else k)
        return self.L.lar_kv_append(self.h, C.byref(self.pages), k, C.byref(self.kv), 4096, 64)

    def read(self, k=None, v=None):
        return self.L.lar_kv_read(self.h, C.byref(self.pages), 4096, 64, C.byref(self.kv if k is None else k),
                                  C.byref(KvRowsArg(1 << 20, 128, 64) if v is None else v))

    def attend(self, q=None):
        return self.L.lar_kv_attend(self.h, C.byref(self.pages), C.byref(self.q if q is None else q), 4096, 64, 0.125,
                                    4096, None)

    def sync(self):
        return self.L.lar_kv_sync(self.h)

    def close(self):
        return self.L.lar_kv_destroy(self.h)


@pytest.mark.parametrize("current", [0, 1])
def test_calls_go_to_the_handles_device(lib, current):
    """A handle made on device 1 works on it whichever device is current, and leaves that one
    current."""
    lib.stub_use(1)
    x = Handle(lib)
    lib.stub_use(current)
    lib.stub_calls(0)
    for call in (lambda: x.plan([1, 5], [40, 100]), x.append, x.read, x.attend, x.sync, x.close):
        lib.stub_calls(1)
        assert call() == 0
        assert lib.stub_device() == current
        assert lib.stub_calls(0) == 0 and lib.stub_calls(1) > 0
