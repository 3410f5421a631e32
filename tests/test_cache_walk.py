"""The chunk kernel's waits for a tile's V, on the CPU: never more than one fill of its
stage ahead of what the waiting block knows, whatever runs a CTA gets."""
import random

import pytest

from tests import cache_walk as W

STAGES = (3, 5, 8)


@pytest.fixture(scope="module")
def lib():
    return W.library()


def _named():
    rng = random.Random(5)
    yield "16 fresh prompts", [1000] * 16, [[1000] * 4] * 16, 7
    yield "fresh prompts, no grouping", [600] * 16, [[600] * 32] * 16, 1
    yield "drafts over heads with budgets", [8] * 64, [[rng.randint(64, 2048) for _ in range(4)] for _ in range(64)], 7
    yield "long and short in turn", [64] * 64, [[2300] * 8, [64] * 8] * 32, 1
    yield "10 tokens, long and short", [10] * 64, [[1500] * 4, [60] * 4] * 32, 7
    yield "more runs than are listed", [5] * 64, [[(5 * b + 7 * h) % 23 for h in range(44)] for b in range(64)], 9


def _count(lib, new, lens, r, v_before_s, **kw):
    ctas = W.runs_of(lib, new, lens, r, **kw)
    return sum(len(W.early_waits(runs, stages, v_before_s)) for stages in STAGES for runs in ctas), ctas


@pytest.mark.parametrize("what,new,lens,r", list(_named()), ids=lambda v: v if isinstance(v, str) else "")
def test_named_batches(lib, what, new, lens, r):
    got, ctas = _count(lib, new, lens, r, lib.w_v_before_s)
    assert got == 0
    # waiting for V first at a run's first tile is what these batches forbid
    if what != "more runs than are listed":
        assert _count(lib, new, lens, r, lambda s, s0: True)[0] > 0
    else:
        assert max(map(len, ctas)) > 16


def test_random_batches(lib):
    rng, wrong = random.Random(6), 0
    for _ in range(300):
        B, H, r = rng.randint(1, 64), rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 7, 8])
        top = 2 ** rng.randint(3, 11)
        new = [rng.randint(0, top) for _ in range(B)]
        lens = [[rng.randint(0, 2 ** rng.randint(3, 13)) if rng.random() < 0.5 else n for _ in range(H)] for n in new]
        kw = dict(workers=rng.choice([1, 20, 152]), causal=rng.randint(0, 1))
        assert _count(lib, new, lens, r, lib.w_v_before_s, **kw)[0] == 0
        wrong += _count(lib, new, lens, r, lambda s, s0: True, **kw)[0] > 0
    assert wrong > 50


def test_runs_cover_every_tile_once(lib):
    new, lens, r = [1000, 37, 0, 300], [[1000, 1400], [37, 40], [5, 5], [299, 9000]], 7
    ctas = W.runs_of(lib, new, lens, r)
    tiles = 0
    for n, heads in zip(new, lens):
        for length in heads:
            for row0 in range(0, n * r, 256):
                end = min(row0 + 256, n * r) - 1
                tiles += -(-max(length - n + end // r + 1, 0) // 128)
    assert sum(s1 - s0 for runs in ctas for s0, s1, _, _ in runs) == tiles
