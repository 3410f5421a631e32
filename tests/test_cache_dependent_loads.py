"""The paged cache's kernels are launched as programmatic dependents, too: pages, lengths,
tables, rows and partial sums may have been written by the kernel before, so none of them is read
by a non-coherent load, and nothing is read ahead of the wait but what the attention kernel's own
wait has seen. From the sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2607_22586_gb300", "csrc")
STARTS = ("cache_start();", "merge_start();")


def _code(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _sources():
    return [n for n in sorted(os.listdir(CSRC)) if n.endswith(".cu") and any(s in _code(n) for s in STARTS)]


def _included(name, seen):
    for inc in re.findall(r'#include "([\w.]+)"', _code(name)):
        if inc not in seen:
            seen.add(inc)
            _included(inc, seen) if os.path.exists(os.path.join(CSRC, inc)) else None
    return seen


def _kernels(code):
    """(name, body) of each __global__ function: from its opening brace to the closing one in column 0."""
    for m in re.finditer(r"__global__[^;{]*?(\w+)\(const __grid_constant__", code):
        body = code[code.index("{\n", m.end()):]
        yield m.group(1), body[:body.index("\n}\n")]


def test_every_kernel_starts_with_a_wait():
    files = _sources()
    assert {"cache.cu", "attend.cu", "attend_token.cu", "attend_umma.cu", "attend_simt.cu"} == set(files)
    names = []
    for f in files:
        code = _code(f)
        assert code.count("__global__") == len(list(_kernels(code))), f
        for name, body in _kernels(code):
            names.append(name)
            assert sum(body.count(s) for s in STARTS) == (2 if name == "attend_merge_row_kernel" else 1), name
    assert len(names) == 7
    # the wait itself comes first in both forms, and whatever is launched behind waits in turn
    start = _code("cache.cuh")
    start = start[start.index("void cache_start()"):]
    assert start.index("griddepcontrol.wait") < start.index("griddepcontrol.launch_dependents")
    merge = _code("attend.cu")
    merge = merge[merge.index("void merge_start()"):]
    assert "griddepcontrol.wait" in merge[:merge.index("}")] and "launch_dependents" not in merge[:merge.index("}")]


def test_no_non_coherent_loads():
    files = _sources()
    headers = set()
    for f in files:
        _included(f, headers)
    assert {"cache.cuh", "attend.cuh", "cache_index.h", "common.cuh", "umma.cuh"} <= headers
    for name in files + [h for h in headers if os.path.exists(os.path.join(CSRC, h)) and h != "common.cuh"]:
        code = _code(name)
        for bad in ("__ldg", "ld.global.nc", "__restrict__", "load_row16("):
            assert bad not in code, (name, bad)


def test_a_merge_reads_only_lengths_ahead_of_its_wait():
    """attend_merge_row_kernel works out which workers share a unit before it waits: from the call's
    description and the lengths, through the L2 (attend_len), which the attention kernel's
    own wait has seen before it let the merge in."""
    body = dict(_kernels(_code("attend.cu")))["attend_merge_row_kernel"]
    ahead = body[:body.index("merge_start();")]
    assert not re.search(r"P\.(po|pml|start)|J\.(kp|vp|ks|vs|table|lens)|A\.(q|out|lse)\b", ahead)
    assert set(re.findall(r"\b(attend_\w+|shares_of|Attend\w+|Parts)\b(?=[ \w]*\()", ahead)) <= {
        "attend_unit", "shares_of", "AttendSums", "Parts"}
    unit = _code("attend.cuh")
    unit = unit[unit.index("int attend_len("):]
    assert "__ldcg(J.lens + u)" in unit[:unit.index("}")]
    for part in ("AttendUnit attend_unit(", "AttendSums(const"):
        text = _code("attend.cuh")
        text = text[text.index(part):]
        text = text[:text.index("\n}" if part.startswith("AttendUnit") else "\n  }")]
        assert "J.lens" not in text and not re.search(r"P\.(po|pml|start)\b", text)
