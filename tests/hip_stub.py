"""Runs a test's code in a process of its own whose library makes its HIP calls to
tests/native/hip_stub.cpp: kernels are noted down and not run.  (A process without
torch, which would find the stub's symbols as well.)"""
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

PRELUDE = f"""
import ctypes, random, sys
sys.modules["torch"] = None
sys.path.insert(0, {os.path.dirname(HERE)!r})
stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import paper_2603_28430_amd as iq
from paper_2603_28430_amd.isoquant import lib


class Launch(ctypes.Structure):
    _fields_ = [("fn", ctypes.c_void_p), ("grid", ctypes.c_uint32 * 3), ("block", ctypes.c_uint32 * 3), ("lds", ctypes.c_uint64)]


def launches():
    '''The launches since the last call, each of which has a kernel and a shape that the device takes.'''
    held = (Launch * 64)()
    n = stub.stub_launches(held, 64)
    assert n <= 64
    for x in held[:n]:
        assert x.fn, "a launch without a kernel"
        assert x.block[0] <= 1024 and x.block[1] == x.block[2] == 1 and x.lds <= 160 * 1024
        assert 0 < x.grid[0] * x.block[0] < 2 ** 32 and 0 < x.grid[1] < 65536 and 0 < x.grid[2] < 65536, list(x.grid)
    return held[:n]
"""


def run(tmp_path, code):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    stub = str(tmp_path / "libhipstub.so")
    subprocess.run([cxx, "-O2", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "native", "hip_stub.cpp"), "-o", stub],
                   check=True, capture_output=True, text=True)
    r = subprocess.run([sys.executable, "-c", PRELUDE + code, stub], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    return r.stdout
