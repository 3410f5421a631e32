"""The prompt kernel's protocol on the host: no wait passes ahead of the phase it means, no role is left
waiting, whichever is slow (tests/prompt_schedule.py; the order of products and the barriers are
csrc/prompt_umma.cu's)."""
import random

import pytest

from tests import prompt_schedule


@pytest.mark.parametrize("stages", [4, 8])         # heads of 128 and of 64
def test_random_runs(stages):
    for seed in range(250):
        rng = random.Random(1000 * stages + seed)
        spec = []
        for _ in range(rng.randrange(1, 12)):
            tiles, two = rng.randrange(1, 5), rng.random() < 0.6
            end0 = max(1, tiles - (rng.random() < 0.4)) if two else tiles
            least = rng.choice([max(1, tiles * 128 - rng.randrange(130)), (tiles - 1) * 128 + 5, 10 ** 9])
            spec.append((tiles, end0, two, least))
        prompt_schedule.simulate(seed, stages, spec)


def test_runs_of_one_block_alone():
    """Blocks in turn, a run each."""
    for stages in (4, 8):
        for seed in range(60):
            prompt_schedule.simulate(seed, stages, [(1 + (seed + i) % 3, 0, False, 1) for i in range(9)])
