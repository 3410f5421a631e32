"""A model of how the chunk kernel's softmax blocks walk their CTA's runs and the ring of
K and V tiles: which fills of the ring a block knows of when it waits for one.

Tile j of a CTA (counted over its runs) has its K at ring position 2j and its V at 2j + 1;
position p lies in stage p % stages, so the fill before it in that stage is p - stages. A
wait by parity tells neighbouring fills apart and no others: it may be made once the fill
before the wanted one is known to be complete. A block knows that positions up to that of
a tile's K are complete once it has waited for the tile's S."""
import ctypes
import os
import shutil
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_22586_gb300", "csrc")

HARNESS = r"""
#include "cache_index.h"
using namespace mmshift;
extern "C" {
int w_keys_of(int causal, int len, int n, int i) { return keys_of(causal, len, n, i); }
long long w_begin(long long W, int most, int i) { return shares_of(W, most, 0).begin(i); }
int w_workers(long long W, int most) { return shares_of(W, most, 0).n; }
int w_v_before_s(int s, int s0) { return v_before_s(s, s0); }
}
"""


def library():
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "needs a host C++ compiler"
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "w.cpp"), os.path.join(tmp, "libwalk.so")
        with open(src, "w") as f:
            f.write(HARNESS)
        subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", so],
                       check=True)
        lib = ctypes.CDLL(so)
    lib.w_begin.restype = ctypes.c_longlong
    lib.w_begin.argtypes, lib.w_workers.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int], [ctypes.c_longlong, ctypes.c_int]
    return lib


def runs_of(lib, new, lens, r, workers=152, causal=1, rows=256, extra=6, extra1=3, few=32, tile=128):
    """The runs of every CTA: [(s0, s1, two blocks, keys that every row attends to)]."""
    widest = max((n * r for n in new if n * r > few), default=0)
    high = min(widest, rows)
    units = []                                         # (pieces, extra, rows, least), in the plan's order
    for n, heads in zip(new, lens):
        if n * r <= few:
            continue
        for length in heads:
            for row0 in range(0, n * r, high):
                m = min(high, n * r - row0)
                keys = lib.w_keys_of(causal, length, n, (row0 + m - 1) // r)
                units.append((-(-keys // tile), extra1 if m <= 128 else extra, m, lib.w_keys_of(causal, length, n, row0 // r)))
    starts, W = [], 0
    for pieces, ex, _, _ in units:
        starts.append(W)
        W += pieces + ex if pieces else 0
    ctas, u = [], 0
    for i in range(lib.w_workers(W, workers) if W else 0):
        begin, end = lib.w_begin(W, workers, i), lib.w_begin(W, workers, i + 1)
        while u + 1 < len(units) and starts[u + 1] <= begin:
            u += 1
        runs, k = [], u
        while k < len(units) and starts[k] < end:
            pieces, ex, m, least = units[k]
            first = starts[k] + ex
            s0, s1 = max(begin, first) - first, max(min(end, first + pieces) - first, 0)
            if pieces and s0 < s1:
                runs.append((s0, s1, m > 128, least))
            k += 1
        ctas.append(runs)
    return ctas


def early_waits(runs, stages, v_before_s, tile=128):
    """Waits of a CTA's blocks for a V whose stage's fill before is not known to be
    complete: [(run, block, fills behind)]."""
    bad = []
    for x in range(2):
        known, j = -1, 0
        for k, (s0, s1, two, least) in enumerate(runs):
            if not two and x != (k & 1):
                j += s1 - s0
                continue
            for s in range(s0, s1):
                masked = s * tile + tile > least
                v = 2 * j + 1
                if not (masked and v_before_s(s, s0)):
                    known = 2 * j                      # S first
                if masked and v - stages > known:
                    bad.append((k, x, (v - stages - known + stages - 1) // stages))
                known = 2 * j
                j += 1
    return bad
