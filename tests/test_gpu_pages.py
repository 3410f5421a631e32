"""Pages shared, copied on writing, compacted and given back, against the pool in plain Python:
tables, counts and lengths have to be equal, and so does every row that a sequence holds."""
import random

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300.cache import PagedKVCache
from tests import cache_ref as R
from tests import pages_ref

pytestmark = pytest.mark.gpu


class Driver:
    """Calls on the pool's tensors and on its plain form, in step."""

    def __init__(self, *a, hq=2, dtype="bf16", seed=0):
        self.P = pages_ref.Pool(*a)
        self.hq, self.dtype = hq * self.P.H, dtype
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        P = self.P
        full = self.shape([P.page * P.max_pages] * P.B)
        self.n = M.mmshift_cache_pages_workspace_size(full, P.struct())
        self.ws = torch.full((self.n + 512,), 0xA5, dtype=torch.uint8, device="cuda")   # only the status word is zero
        self.ws[:256].zero_()

    def shape(self, new, stride=0):
        P = self.P
        return M.make_shape(self.hq, P.H, P.d, 2, 0 if self.dtype == "bf16" else 1, R.cu_of(new), [1] * P.B, n_layers=P.L,
                            layer_stride_kv=stride)

    def append(self, new):
        P, T = self.P, sum(new)
        k, v = (torch.randn((P.L, T, P.H, P.d), generator=self.gen, device="cuda").to(R.DT[self.dtype]) for _ in range(2))
        P.lens.add_(torch.tensor(new, dtype=torch.int32, device="cuda")[None, :, None])
        s = self.shape(new, T * P.H * P.d)
        M.check(M.mmshift_cache_reserve(s, P.struct(), P.refs, self.ws, self.n), "reserve")
        M.check(M.mmshift_cache_append(s, P.struct(), k, v, 0, self.ws, self.n), "append")
        P.reserve(new, P.lens.tolist())
        cu = R.cu_of(new)
        for l, b, h in P.units():
            P.append(l, b, h, k[l, cu[b]:cu[b + 1], h], v[l, cu[b]:cu[b + 1], h])

    def fork(self, src, dst):
        P = self.P
        M.check(M.mmshift_cache_fork(self.shape([0] * P.B), P.struct(), P.refs, src, dst, self.ws, self.n), "fork")
        P.fork(src, dst)

    def free(self, which):
        P = self.P
        M.check(M.mmshift_cache_free(self.shape([0] * P.B), P.struct(), P.refs, which, self.ws, self.n), "free")
        P.release(which)

    def compact(self, rows, idx=None, counts=None, rng=None):
        P, cu = self.P, R.cu_of(rows)
        if idx is None:
            idx = torch.full((P.L, cu[-1], P.H), -1, dtype=torch.int32)
            for l, b, h in P.units():
                held = len(P.held[l][b][h])
                m = min(rows[b], held)
                idx[l, cu[b]:cu[b] + m, h] = torch.tensor(sorted(rng.sample(range(held), m)), dtype=torch.int32)
        c = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        M.check(M.mmshift_cache_compact(self.shape(rows), P.struct(), P.refs, idx.cuda(), c, self.ws, self.n), "compact")
        P.compact(idx.tolist(), rows, counts)

    def poll(self):
        assert (self.ws[self.n:] == 0xA5).all()
        return M.mmshift_poll_status(self.ws)


@pytest.mark.parametrize("dtype,kind,d,page", [("bf16", "bf16", 128, 64), ("bf16", "i8", 128, 16), ("f32", "f32", 64, 32),
                                               ("f32", "i8", 64, 256), ("bf16", "bf16", 64, 16), ("f32", "f32", 128, 128)])
def test_a_life_of_a_pool(dtype, kind, d, page):
    D = Driver(2, 5, 2, d, kind, page, 220, 700 // page + 2, dtype=dtype)
    rng = random.Random(3)
    D.append([page + 3, 0, 1, 2 * page, 0])
    D.P.check("first")
    D.fork([0, 3], [1, 4])
    D.P.check("fork")
    D.append([1, 1, 1, 0, 5])                      # tails are copied; 3 and 4 write where nobody else does
    D.P.check("copies")
    D.fork([1, 1, 1], [0, 2, 3])                   # what they held is given back, a source of three
    D.append([0, page, 1, 2, 300 if page < 256 else 30])
    D.P.check("three")
    D.compact([0, page // 2, 3, 0, page + 5], rng=rng)
    D.P.check("compact")
    D.append([4, 4, 4, 4, 4])
    D.free([1])
    D.P.check("free")
    D.append([0, 7, 0, 0, 1])
    D.compact([2, 2, 2, 2, 2], rng=rng)
    D.P.check("short")
    D.free([0, 1, 2, 3, 4])
    D.P.check("empty")
    assert D.poll() == M._lib.MMSHIFT_OK
    assert not D.P.refs.any() and (D.P.table == -1).all()


@pytest.mark.parametrize("kind,d,rows,keep", [("bf16", 128, 1500, 900), ("i8", 64, 2100, 2099), ("f32", 128, 700, 1), ("bf16", 64, 1111, 1111)])
def test_compaction_of_long_sequences(kind, d, rows, keep):
    """Many chunks of rows, one sequence's by a cluster and several's by a block each."""
    for B, H in ((1, 1), (9, 5)):
        n = rows if B == 1 else min(rows, 500)
        m = min(keep, n)
        D = Driver(1, B, H, d, kind, 16, B * H * (n // 16 + 2), n // 16 + 2, dtype="f32" if kind == "f32" else "bf16")
        D.append([n] * B)
        D.compact([m] * B, rng=random.Random(5))
        D.P.check((B, H))
        assert D.poll() == M._lib.MMSHIFT_OK


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("i8", 128), ("f32", 64)])
@pytest.mark.parametrize("L,B,H", [(1, 4, 7), (3, 3, 9), (2, 5, 5)])
def test_compaction_by_few_blocks_a_sequence(kind, d, L, B, H):
    """Four blocks a sequence, two, and four of layers; lengths that differ, one empty."""
    D = Driver(L, B, H, d, kind, 16, L * B * H * 44, 44, hq=1, dtype="f32" if kind == "f32" else "bf16")
    lens = [[643, 0, 300, 129, 64], [500, 431, 17, 1, 256]][B % 2][:B]
    D.append(lens)
    D.compact([n * 2 // 3 for n in lens], rng=random.Random(7))
    D.P.check((L, B, H))
    assert D.poll() == M._lib.MMSHIFT_OK


def test_shared_pages_are_not_compacted_in_place():
    D = Driver(1, 3, 2, 64, "bf16", 16, 60, 9)
    D.append([100, 0, 0])
    D.fork([0, 0], [1, 2])
    D.compact([0, 50, 33], rng=random.Random(1))
    D.P.check("two of three")
    D.compact([40, 0, 0], rng=random.Random(2))    # by now its pages are its own
    D.P.check("the last")
    assert D.poll() == M._lib.MMSHIFT_OK


def test_counts_keep_fewer_rows_of_a_head():
    D = Driver(2, 2, 3, 64, "f32", 16, 80, 5, dtype="f32")
    D.append([60, 30])
    counts = [[[0, 1, 40], [16, 30, 31]], [[60, 61, 17], [2 ** 31 - 1, -5, 3]]]
    idx = torch.arange(40, dtype=torch.int32)[:, None].expand(40, 3)
    idx = torch.cat([idx, idx[:30]])[None].expand(2, 70, 3).contiguous()
    D.compact([40, 30], idx=idx, counts=counts)
    D.P.check("counts")
    assert D.poll() == M._lib.MMSHIFT_OK


def test_bad_indices_give_zero_rows():
    D = Driver(1, 1, 1, 64, "bf16", 16, 12, 6)
    D.append([70])
    idx = torch.tensor([0, 0, 2, 69, 70, 2 ** 31 - 1, -1, -2 ** 31, 8, 8, 60], dtype=torch.int32)[None, :, None]
    D.compact([11], idx=idx)
    D.P.check("zeros")
    assert D.poll() == M._lib.MMSHIFT_ERR_DEVICE and D.poll() == M._lib.MMSHIFT_OK


def test_no_page_free():
    """Sequences that got none lose what the page held, others nothing."""
    D = Driver(1, 3, 1, 64, "bf16", 16, 5, 4)
    D.append([40, 0, 0])
    D.fork([0, 0], [1, 2])
    D.append([1, 1, 1])                            # three copies of the tail, two pages free
    assert D.P.exhausted
    D.P.check("two copies")
    assert D.poll() == M._lib.MMSHIFT_ERR_DEVICE
    D.free([1])
    D.P.check("freed")
    D.P.exhausted = False
    D.append([3, 9, 0])
    assert not D.P.exhausted
    D.P.check("again")
    assert D.poll() == M._lib.MMSHIFT_OK


def test_rows_behind_the_table():
    D = Driver(1, 2, 1, 64, "bf16", 16, 9, 2)
    D.append([30, 1])
    D.P.lens.add_(torch.tensor([10, 1], dtype=torch.int32, device="cuda")[None, :, None])
    s = D.shape([10, 1])
    M.check(M.mmshift_cache_reserve(s, D.P.struct(), D.P.refs, D.ws, D.n), "reserve")
    D.P.reserve([10, 1], D.P.lens.tolist())
    assert D.P.table.tolist() == D.P.m_table and D.P.refs.tolist() == D.P.m_refs
    D.P.lens.fill_(2 ** 31 - 1)                    # no length: the table's end, as in append
    M.check(M.mmshift_cache_reserve(s, D.P.struct(), D.P.refs, D.ws, D.n), "reserve")
    D.P.reserve([10, 1], D.P.lens.tolist())
    assert D.P.table.tolist() == D.P.m_table and D.P.refs.tolist() == D.P.m_refs
    assert D.poll() == M._lib.MMSHIFT_OK


def test_many_sequences_and_pages():
    """More sequences than the cluster has threads, and a pool of which each warp scans thousands."""
    D = Driver(20, 64, 8, 64, "i8", 16, 300000, 4)
    P = D.P
    used = torch.randperm(300000, generator=torch.Generator().manual_seed(1))[:200000]
    P.refs[used.cuda()] = 1                        # held by other sequences
    for new in ([1] * 64, [0, 17] * 32):
        before, refs = P.table.clone(), P.refs.clone()
        P.lens.add_(torch.tensor(new, dtype=torch.int32, device="cuda")[None, :, None])
        M.check(M.mmshift_cache_reserve(D.shape(new), P.struct(), P.refs, D.ws, D.n), "reserve")
        first = torch.arange(4, device="cuda") * 16
        need = (first < P.lens[..., None]) & (before < 0) & (torch.tensor(new, device="cuda") > 0)[None, :, None, None]
        free = (refs == 0).nonzero()[:int(need.sum()), 0].int()
        before[need] = free
        refs[free.long()] = 1
        assert torch.equal(P.table, before) and torch.equal(P.refs, refs)
    assert D.poll() == M._lib.MMSHIFT_OK


def test_captured_steps():
    """A captured advance and append, replayed while the sequences grow and copy their tails."""
    D = Driver(2, 4, 2, 64, "bf16", 16, 120, 8)
    P = D.P
    D.append([20, 0, 0, 0])
    D.fork([0, 0, 0], [1, 2, 3])
    new, s = [1] * 4, D.shape([1] * 4, 4 * 2 * 64)
    k, v = (torch.zeros((2, 4, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    one = torch.ones((1, 4, 1), dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        P.lens.add_(one)
        M.check(M.mmshift_cache_reserve(s, P.struct(), P.refs, D.ws, D.n, torch.cuda.current_stream()), "reserve")
        M.check(M.mmshift_cache_append(s, P.struct(), k, v, 0, D.ws, D.n, torch.cuda.current_stream()), "append")
    for step in range(30):
        for x in (k, v):
            x.copy_(torch.randn(x.shape, generator=D.gen, device="cuda").to(x.dtype))
        graph.replay()
        P.reserve(new, P.lens.tolist())
        for l, b, h in P.units():
            P.append(l, b, h, k[l, b:b + 1, h], v[l, b:b + 1, h])
        if step in (0, 11, 12, 29):
            P.check(step)
    assert D.poll() == M._lib.MMSHIFT_OK


def test_random_lives():
    """Forks, growth, compactions and releases in any order."""
    for seed in range(6):
        rng = random.Random(seed)
        B, H, L = rng.choice([1, 3, 8]), rng.choice([1, 2, 5]), rng.choice([1, 3])
        page = rng.choice([16, 32])
        D = Driver(L, B, H, 64, rng.choice(["bf16", "i8"]), page, L * B * H * 8 + 3, 8, seed=seed)
        for step in range(14):
            kind = rng.choice(["append", "append", "fork", "compact", "free"])
            lens = [max(len(D.P.held[l][b][h]) for l in range(L) for h in range(H)) for b in range(B)]
            if kind == "append":
                D.append([rng.choice([0, 1, 2, page, 40]) if lens[b] < 8 * page - 40 else 0 for b in range(B)])
            elif kind == "fork" and B > 1:
                src = rng.randrange(B)
                dst = rng.sample([b for b in range(B) if b != src], rng.randrange(1, B))
                D.fork([src] * len(dst), dst)
            elif kind == "compact":
                D.compact([rng.choice([0, rng.randrange(lens[b] + 1)]) for b in range(B)], rng=rng)
            elif kind == "free":
                D.free(rng.sample(range(B), rng.randrange(B + 1)))
            if not D.P.exhausted:
                D.P.check((seed, step, kind))
            else:
                break


def test_the_class():
    """PagedKVCache with a pool: fill, advance, fork, attend, compact and free through the methods."""
    from paper_2607_22586_gb300.selector import KVSelector

    gen = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    sel = KVSelector(6, 2, 64, 8, torch.bfloat16, [0, 200, 290], [50, 30], n_layers=2,
                     params=M.default_params(n_proxies=32, n_groups=2))
    K, V, Q = rnd(2, 290, 2, 64), rnd(2, 290, 2, 64), rnd(2, 2, 8, 6, 64)
    idx, kk, vv = sel(K, V, Q)
    cache = PagedKVCache(6, 2, 64, torch.bfloat16, 2, 100, n_layers=2, page_size=16, pages=60)
    own = PagedKVCache(6, 2, 64, torch.bfloat16, 2, 100, n_layers=2, page_size=16)
    for c in (cache, own):
        c.fill(sel, K, V)
    used = int((cache.refs > 0).sum())
    assert used == 2 * 2 * (4 + 2) and cache.lens.tolist() == own.lens.tolist()
    for new in ([3, 1], [17, 0]):
        q, k, v = rnd(2, sum(new), 6, 64), rnd(2, sum(new), 2, 64), rnd(2, sum(new), 2, 64)
        for c in (cache, own):
            c.advance(new)
            c.append(k, v, new)
        for layer in range(2):
            a, b = (c.attend(q[layer], new, layer) for c in (cache, own))
            assert R.same(a, b)
    for x, y in zip(cache.read([70, 31]), own.read([70, 31])):
        assert R.same(x, y)
    cache.fork([0], [1])
    keep = torch.arange(0, 60, 2, dtype=torch.int32, device="cuda")[None, :, None].expand(2, 30, 2).contiguous()
    k0, _ = cache.read([70, 70])
    cache.compact(keep, [0, 30])
    k1, _ = cache.read([70, 30])
    assert R.same(k1[:, :70], k0[:, :70]) and R.same(k1[:, 70:], k0[:, 0:60:2])
    cache.free([0, 1])
    assert not cache.refs.any()
    cache.poll()
    for bad in (lambda: own.fork([0], [1]), lambda: own.free([0]), lambda: cache.fork([0], [2]), lambda: cache.free([-1]),
                lambda: cache.compact(keep, [0, 31]), lambda: cache.compact(keep.long(), [0, 30])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cache.fork([0], [0]), lambda: cache.fork([0, 0], [1, 1]), lambda: cache.fork([0, 1], [1, 0])):
        with pytest.raises(M.MMShiftError):
            bad()


def test_compaction_without_free_pages():
    """Rows whose shared pages nothing can replace are lost; the other holder keeps them."""
    D = Driver(1, 2, 1, 64, "f32", 16, 5, 4, dtype="f32")
    D.append([60, 0])
    D.fork([0], [1])
    D.compact([0, 40], rng=random.Random(4))       # three pages wanted, one free
    assert D.P.exhausted
    D.P.check("first page kept")
    assert D.poll() == M._lib.MMSHIFT_ERR_DEVICE
    D.free([0])
    D.P.check("freed")
    assert D.poll() == M._lib.MMSHIFT_OK


def test_pages_past_four_gigabytes():
    """Sequences whose pages are the pool's last."""
    D = Driver(1, 2, 1, 128, "f32", 256, 36000, 4, dtype="f32")
    P = D.P
    assert (P.n_pages - 12) * 256 * 128 * 4 > 2 ** 32
    P.refs[:P.n_pages - 12] = 1                    # held by others
    P.m_refs[:P.n_pages - 12] = [1] * (P.n_pages - 12)
    D.append([700, 0])
    D.fork([0], [1])
    D.append([3, 300])
    D.compact([0, 450], rng=random.Random(6))
    D.compact([333, 0], rng=random.Random(7))
    assert P.table[P.table >= 0].min() >= P.n_pages - 12 and not P.exhausted
    P.check("last pages")
    assert D.poll() == M._lib.MMSHIFT_OK


def state(D, what=""):
    """Tables, counts and lengths; rows of lost pages are not known, so none are compared."""
    P = D.P
    assert P.table.tolist() == P.m_table, (what, "table")
    assert P.refs.tolist() == P.m_refs, (what, "refs")
    assert P.lens.tolist() == [[[len(x) for x in y] for y in z] for z in P.held], (what, "lens")
    # the counts are the entries that name a page, whatever was lost
    named = P.table[P.table >= 0].long().flatten()
    assert torch.equal(P.refs.long(), torch.bincount(named, minlength=P.n_pages)), (what, "entries")


def emptied(D):
    D.free(range(D.P.B))
    state(D, "emptied")
    assert not D.P.refs.any() and (D.P.table == -1).all()
    D.poll()


@pytest.mark.parametrize("n_pages", [2, 3, 4, 9])
def test_more_pages_wanted_than_the_pool_has(n_pages):
    """Every holder of a shared page writes to it, and the pool is smaller than their number."""
    D = Driver(1, 8, 1, 64, "bf16", 16, n_pages, 4)
    D.append([20] + [0] * 7)
    D.fork([0] * 7, range(1, 8))
    D.append([1] * 8)
    assert D.P.exhausted
    D.P.check("copies of the tail")
    state(D, "copies of the tail")
    assert D.poll() == M._lib.MMSHIFT_ERR_DEVICE
    emptied(D)
    D.append([0, 16 * min(n_pages, 4)] + [0] * 6)  # every page is there again
    D.P.check("again")
    assert D.poll() == M._lib.MMSHIFT_OK


@pytest.mark.parametrize("L,B,H,rows,keep,max_pages,n_pages", [
    (1, 3, 1, 60, 40, 4, 5),              # one block, a lane a sequence
    (1, 2, 1, 2200, 2150, 140, 140),      # more pages of a sequence than its lanes hold at once
    (3, 40, 20, 90, 50, 6, 1000),         # a cluster of blocks
])
def test_compaction_that_wants_more_pages_than_the_pool_has(L, B, H, rows, keep, max_pages, n_pages):
    D = Driver(L, B, H, 64, "bf16", 16, n_pages, max_pages)
    D.append([rows] + [0] * (B - 1))
    assert not D.P.exhausted
    D.fork([0] * (B - 1), range(1, B))
    counts = None
    if B == 3:
        counts = [[[40], [17], [33]]]
    idx = torch.arange(rows - keep, rows, dtype=torch.int32).repeat(B)[None, :, None].expand(L, B * keep, H).contiguous()
    D.compact([keep] * B, idx=idx, counts=counts)
    assert D.P.exhausted and sum(p < 0 for x in D.P.m_table for y in x for z in y for p in z[:1]) > 0
    state(D, "compacted")
    assert D.poll() == M._lib.MMSHIFT_ERR_DEVICE
    emptied(D)


def test_many_sequences_of_a_small_pool():
    """More sequences than the cluster has threads, each of which wants a page of its own."""
    D = Driver(17, 64, 8, 64, "i8", 16, 400, 3)
    P = D.P
    for new, copies in (([20] + [0] * 63, True), ([1] * 64, False), ([0, 30] * 32, False)):
        lens = P.lens + torch.tensor(new, dtype=torch.int32, device="cuda")[None, :, None]
        P.lens.copy_(lens)
        M.check(M.mmshift_cache_reserve(D.shape(new), P.struct(), P.refs, D.ws, D.n), "reserve")
        P.reserve(new, lens.tolist())
        for l, b, h in P.units():
            P.held[l][b][h] += [None] * new[b]
        state(D, new[:2])
        if copies:
            D.fork([0] * 63, range(1, 64))
    assert P.exhausted and D.poll() == M._lib.MMSHIFT_ERR_DEVICE
    emptied(D)


def test_random_lives_of_pools_that_are_too_small():
    """As the lives above, on past every page that was not there."""
    exhausted = 0
    for seed in range(8):
        rng = random.Random(100 + seed)
        B, H, L = rng.choice([3, 8]), rng.choice([1, 2, 5]), rng.choice([1, 3])
        n_pages = rng.choice([3, L * H, L * H * B])
        D = Driver(L, B, H, 64, rng.choice(["bf16", "i8"]), 16, n_pages, 8, seed=seed)
        for step in range(16):
            kind = rng.choice(["append", "append", "fork", "fork", "compact", "free"])
            lens = [max(len(D.P.held[l][b][h]) for l in range(L) for h in range(H)) for b in range(B)]
            if kind == "append":
                D.append([rng.choice([0, 1, 2, 16, 40]) if lens[b] < 8 * 16 - 40 else 0 for b in range(B)])
            elif kind == "fork":
                src = rng.randrange(B)
                dst = rng.sample([b for b in range(B) if b != src], rng.randrange(1, B))
                D.fork([src] * len(dst), dst)
            elif kind == "compact":
                D.compact([rng.choice([0, rng.randrange(lens[b] + 1)]) for b in range(B)], rng=rng)
            else:
                D.free(rng.sample(range(B), rng.randrange(2)))
            state(D, (seed, step, kind))
        exhausted += D.P.exhausted
        emptied(D)
    assert exhausted > 4


def test_a_fill_whose_counts_are_the_lengths():
    """As many rows of another selection as the sequences hold already."""
    from paper_2607_22586_gb300.selector import KVSelector

    gen = torch.Generator(device="cuda").manual_seed(8)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    sel = KVSelector(6, 2, 64, 8, torch.bfloat16, [0, 200, 290], [50, 30], n_layers=2,
                     params=M.default_params(n_proxies=32, n_groups=2))
    K, V, Q = rnd(2, 290, 2, 64), rnd(2, 290, 2, 64), rnd(2, 2, 8, 6, 64)
    sel(K, V, Q)
    counts = torch.tensor([[[50, 1], [0, 30]], [[17, 33], [29, 64]]], dtype=torch.int32, device="cuda")
    held = counts.clamp(max=torch.tensor([50, 30], dtype=torch.int32, device="cuda")[None, :, None])
    read = []
    for pages in (60, None):
        cache = PagedKVCache(6, 2, 64, torch.bfloat16, 2, 100, n_layers=2, page_size=16, pages=pages)
        cache.lens.copy_(counts if pages is None else 0)
        if pages is not None:
            cache.fill(sel, K, V, counts=counts)
        cache.fill(sel, K, V, counts=cache.lens)
        assert cache.lens.tolist() == held.tolist()
        read.append(cache.read([50, 30]))
        cache.poll()
    for x, y in zip(*read):
        assert R.same(x, y)
