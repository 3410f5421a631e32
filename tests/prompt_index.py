"""The order in which prompts' units are shared out, compiled for the host."""
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_22586_gb300", "csrc")

SOURCE = r"""
#include "prompt_index.h"
using namespace mmshift;
extern "C" int order(int B, const int32_t* off, int r, int rows, int heads, int causal, int workers, int start, int merge,
                     int32_t* unit, int32_t* turn, int most) {
  const PromptOrder O = prompt_order(B, off, r, rows, heads, causal);
  for (int i = 0; i < O.units && i < most; ++i) {
    const PromptUnit u = prompt_unit(O, heads, causal, i);
    unit[4 * i] = u.b;
    unit[4 * i + 1] = u.h;
    unit[4 * i + 2] = u.tile;
    unit[4 * i + 3] = prompt_tile_keys(off[u.b + 1] - off[u.b], r, rows, causal, u.tile);
  }
  for (int w = 0; w < workers; ++w)
    for (int k = 0; k * workers < O.units; ++k) {
      const int u = prompt_turn(O, workers, w, k);
      if (u >= 0 && u < most) turn[u] += 1;
    }
  return O.units | (prompt_whole(O, off, r, rows, heads, causal, workers, start, merge) ? 1 << 30 : 0);
}
"""


def library(tmp):
    src, so = os.path.join(tmp, "prompt_index.cc"), os.path.join(tmp, "prompt_index.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-I", CSRC, src, "-o", so])
    return ctypes.CDLL(so)
