"""csrc/cache_index.h through the host C++ compiler, as a ctypes library."""
import ctypes
import os
import shutil
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_22586_gb300", "csrc")

HARNESS = r"""
#include "cache_index.h"
using namespace mmshift;
extern "C" {
int t_range_of(const int32_t* off, int n, int x) { return range_of(off, n, x); }
int t_page_row(int page, int n_pages, int shift, int t) { return page_row(page, n_pages, shift, t); }
int t_keys_of(int causal, int len, int n, int i) { return keys_of(causal, len, n, i); }
long long t_span_begin(long long W, int n, int i) { return span_begin(W, n, i); }
int t_span_of(long long W, int n, long long x) { return span_of(W, n, x); }
int t_span_workers(long long W, int most, int least) { return span_workers(W, most, least); }
}
"""


def library():
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "needs a host C++ compiler"
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "i.cpp"), os.path.join(tmp, "libindex.so")
        with open(src, "w") as f:
            f.write(HARNESS)
        subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", so],
                       check=True)
        lib = ctypes.CDLL(so)
    lib.t_span_begin.restype = ctypes.c_longlong
    lib.t_span_begin.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    lib.t_span_of.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong]
    lib.t_span_workers.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return lib
