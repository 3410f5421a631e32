"""Every unit of a batch of prompts is somebody's, once, longest first, on the host."""
import ctypes
import random

import pytest

from tests import prompt_index


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return prompt_index.library(str(tmp_path_factory.mktemp("prompt_index")))


def order(lib, lens, r, rows, heads, causal, workers=152, start=2, merge=6):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    tiles = [(n * r + rows - 1) // rows for n in lens]
    total = sum(tiles) * heads
    unit, turn = (ctypes.c_int32 * (4 * total + 4))(), (ctypes.c_int32 * (total + 1))()
    got = lib.order(len(lens), (ctypes.c_int32 * len(off))(*off), r, rows, heads, causal, workers, start, merge, unit, turn, total)
    assert got & ~(1 << 30) == total
    return [tuple(unit[4 * i:4 * i + 4]) for i in range(total)], list(turn[:total]), bool(got >> 30 & 1), tiles


@pytest.mark.parametrize("causal", [0, 1])
def test_units(lib, causal):
    rng = random.Random(5)
    for trial in range(60):
        lens = [rng.choice([0, 1, 17, 36, 37, 128, rng.randrange(1, 3000)]) for _ in range(rng.choice([1, 2, 5, 16, 64]))]
        if not any(lens):
            continue
        r, heads = rng.choice([(1, 3), (7, 4), (8, 8), (40, 1), (130, 2)])
        block = 128 // r * r if r <= 128 else 128
        rows = min(2 * block, max(lens) * r)
        units, turn, whole, tiles = order(lib, lens, r, rows, heads, causal, workers=rng.choice([1, 7, 152]))
        want = {(b, h, t) for b, n in enumerate(tiles) for h in range(heads) for t in range(n)}
        assert {u[:3] for u in units} == want and len(units) == len(want)
        assert turn == [1] * len(units)
        for b, h, t, keys in units:
            last = min((t + 1) * rows, lens[b] * r) - 1
            assert keys == (last // r + 1 if causal else lens[b])
        # longest first, but for the last, shorter tile of a request
        key = [u[2] if causal else lens[u[0]] for u in units]
        assert key == sorted(key, reverse=True)


def test_when_units_are_shared(lib):
    assert order(lib, [32768], 7, 252, 4, 1)[2]                 # 24 units a worker
    assert order(lib, [1036, 529, 2116, 37], 1, 256, 16, 0)[2]
    assert order(lib, [17], 7, 119, 4, 1)[2]
    assert not order(lib, [4096], 7, 252, 1, 0)[2]              # 114 units of 32 tiles: a quarter of the workers idle
    assert not order(lib, [8000], 8, 256, 8, 0, workers=1500)[2]
