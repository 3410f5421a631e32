"""Index arithmetic of the paged cache on the CPU: bad table entries, empty
requests, rows without keys, and the shares of attention's workers."""
import ctypes
import random

import pytest

from tests import cache_index


@pytest.fixture(scope="module")
def lib():
    return cache_index.library()


def test_request_of_a_row(lib):
    rng = random.Random(1)
    for _ in range(300):
        lens = [rng.choice([0, 0, 1, 2, 7, 100]) for _ in range(rng.randint(1, 64))]
        off = [0]
        for n in lens:
            off.append(off[-1] + n)
        arr = (ctypes.c_int32 * len(off))(*off)
        want = [b for b, n in enumerate(lens) for _ in range(n)]
        assert [lib.t_range_of(arr, len(lens), x) for x in range(off[-1])] == want


@pytest.mark.parametrize("shift", [4, 5, 6, 7, 8])
def test_position_in_the_pool(lib, shift):
    page = 1 << shift
    n_pages = (2 ** 31 - 1 - 256) // page
    for bad in (-1, -2 ** 31, n_pages, 2 ** 31 - 1):
        assert lib.t_page_row(bad, n_pages, shift, 5) == -1
    for p in (0, 1, n_pages - 1):
        for t in (0, 1, page - 1, page, 7 * page + 3, 2 ** 30 - 1):
            assert lib.t_page_row(p, n_pages, shift, t) == p * page + t % page >= 0


def test_keys_of_a_token(lib):
    for length in range(6):
        for n in range(1, 6):
            for i in range(n):
                assert lib.t_keys_of(1, length, n, i) == max(0, length - (n - 1 - i))
                assert lib.t_keys_of(0, length, n, i) == length


def test_shares_cover_all_work_once(lib):
    rng = random.Random(2)
    for _ in range(400):
        W, most, least = rng.choice([1, 2, 151, 152, 1000, rng.randint(1, 3000)]), rng.choice([1, 2, 152, 456]), rng.choice([0, 2])
        n = lib.t_workers(W, most, least)
        assert n == max(1, min(most, -(-W // 2 ** least)))
        begins = [lib.t_begin(W, most, least, i) for i in range(n + 1)]
        assert begins[0] == 0 and begins[-1] == W
        sizes = [b - a for a, b in zip(begins, begins[1:])]
        assert max(sizes) - min(sizes) <= 1 and min(sizes) >= 1
        owner = [i for i, s in enumerate(sizes) for _ in range(s)]
        assert [lib.t_of(W, most, least, x) for x in range(W)] == owner
    for big in (2 ** 31 - 1, 2 ** 32 + 7, 2 ** 40):      # pieces past 32 bits
        for x in (0, 1, 2 ** 31 - 5, big - 1):
            i = lib.t_of(big, 456, 0, x)
            assert lib.t_begin(big, 456, 0, i) <= x < lib.t_begin(big, 456, 0, i + 1)


def test_no_work_has_one_worker(lib):
    assert lib.t_workers(0, 152, 2) == 1
    assert lib.t_begin(0, 152, 2, 1) == 0


def test_quotients(lib):
    rng = random.Random(3)
    for _ in range(2000):
        x, y = rng.randrange(2 ** rng.randint(1, 62)), 1 + rng.randrange(2 ** rng.randint(1, 40))
        assert lib.t_quotient(x, y) == x // y


def test_division_by_a_known_number(lib):
    rng = random.Random(4)
    ds = list(range(1, 130)) + [2 ** k + e for k in range(1, 31) for e in (-1, 0, 1) if 2 ** k + e <= 2 ** 31 - 1]
    for d in ds:
        xs = [0, 1, d - 1, d, d + 1, 2 ** 31 - 1, 2 ** 31 - 2, (2 ** 31 - 1) // d * d, (2 ** 31 - 1) // d * d - 1]
        xs += [rng.randrange(2 ** 31) for _ in range(20)]
        for x in xs:
            if 0 <= x < 2 ** 31:
                assert lib.t_divide(d, x) == x // d, (d, x)
