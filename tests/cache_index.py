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
long long t_begin(long long W, int most, int least, int i) { return shares_of(W, most, least).begin(i); }
int t_of(long long W, int most, int least, long long x) { return shares_of(W, most, least).of(x); }
int t_workers(long long W, int most, int least) { return shares_of(W, most, least).n; }
int t_divide(int d, int x) { return divisor_of(d)(x); }
long long t_quotient(long long x, long long y) { return quotient(x, y); }
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
    ll, i = ctypes.c_longlong, ctypes.c_int
    lib.t_begin.restype = lib.t_quotient.restype = ll
    lib.t_begin.argtypes, lib.t_of.argtypes, lib.t_workers.argtypes = [ll, i, i, i], [ll, i, i, ll], [ll, i, i]
    lib.t_quotient.argtypes = [ll, ll]
    return lib
