"""Registers are given up and taken by whole warpgroups (PTX: all warps of one execute the same setmaxnreg, and
none lies in a branch that they do not take together), and no more are taken than the launch has. From the
sources."""
import os
import re

from tests.test_cache_dependent_loads import CSRC, _code

CHANGE = re.compile(r"setmaxnreg\.(inc|dec)")


def test_warpgroups_change_their_registers_as_wholes():
    files = [f for f in sorted(os.listdir(CSRC)) if f.endswith((".cu", ".cuh", ".h")) and CHANGE.search(_code(f))]
    assert files == ["prompt_umma.cu"]
    code = _code(files[0])
    assert sorted(CHANGE.findall(code)) == ["dec", "inc"]
    roles = {name: int(first) for name, first in re.findall(r"\b([A-Z]+) = (\d+)", code[code.index("PRODUCER = "):code.index("FINISHER = ") + 20])}
    assert roles["PRODUCER"] % 4 == 0 and roles["PRODUCER"] == min(roles.values())
    # one branch at the kernel's outermost level, each side of which begins with its change
    one = re.findall(r"\n  if \(warp >= PRODUCER\) \{\n    fewer_registers\(\);\n", code)
    other = re.findall(r"\n  \} else \{\n    more_registers\(\);\n", code)
    assert len(one) == len(other) == 1
    assert code.count("fewer_registers()") == code.count("more_registers()") == 2      # the function, and that call
    split = dict(re.findall(r"\b(SOFTMAX_REGS|OTHER_REGS) = (\d+)", code))
    assert 256 * sum(map(int, split.values())) <= 512 * 128
