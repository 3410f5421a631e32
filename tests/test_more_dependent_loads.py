"""Kernels launched as programmatic dependents beside the cache's: their start waits for everything
before, and what was written there is read by no non-coherent load. From the sources."""
import os

from tests.test_cache_dependent_loads import CSRC, _code, _included, _kernels

STARTS = {"pages.cu": "pages_start", "shared.cu": "shared_start", "rope.cu": "rope_start",
          "prompt_umma.cu": "prompt_start"}


def test_every_kernel_waits_before_it_reads():
    for name, start in STARTS.items():
        code = _code(name)
        kernels = list(_kernels(code))
        assert code.count("__global__") == len(kernels) > 0, name
        for kernel, body in kernels:
            assert body.count(start + "();") == 1, (name, kernel)
            ahead = body[:body.index(start + "();")]
            for bad in ("J.lens", "J.table", "G.refs", "G.table", "J.pos", "sum_of_row", "cache_len", "load", "attend_span"):
                assert bad not in ahead, (name, kernel, bad)
        wait = code[code.index(f"void {start}()"):]
        wait = wait[:wait.index("\n}")]
        assert wait.index("griddepcontrol.wait") < wait.index("griddepcontrol.launch_dependents"), name


def test_no_non_coherent_loads():
    for name in STARTS:
        for f in [name] + [h for h in _included(name, set()) if os.path.exists(os.path.join(CSRC, h)) and h != "common.cuh"]:
            for bad in ("__ldg", "ld.global.nc", "__restrict__", "load_row16("):
                assert bad not in _code(f), (f, bad)
