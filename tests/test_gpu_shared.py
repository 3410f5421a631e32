"""Attention over sequences that share pages: what mmshift_cache_attention gives, by the same formula and
bounds (and 16 roundings more, of the joining)."""
import math

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300.cache import PagedKVCache
from tests import cache_ref as R

pytestmark = pytest.mark.gpu


def share(cache, groups, common):
    """The first request's pages of the first `common[g]` pages, for all requests of a group."""
    b0 = 0
    for g, n in enumerate(groups):
        for b in range(b0 + 1, b0 + n):
            for h in range(cache.H):
                c = common[g] if isinstance(common[g], int) else common[g][h]
                cache.table[0, b, h, :c] = cache.table[0, b0, h, :c]
        b0 += n
    return cache


def attend(cache, q, new, groups, causal=True, scale=0.0, status=M._lib.MMSHIFT_OK, stride=0, lse=True):
    struct, cu = cache.struct(0), R.cu_of(groups)
    shape = R.shape_of(cache, new, q.shape[1], "bf16" if q.dtype == torch.bfloat16 else "f32", layers=1)
    n = M.mmshift_cache_shared_workspace_size(shape, struct, cu)
    ws = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    ws[:256].zero_()
    out = torch.full(q.shape, math.nan, dtype=q.dtype, device="cuda")
    ls = torch.full(q.shape[:2], math.nan, device="cuda") if lse else None
    M.check(M.mmshift_cache_attention_shared(shape, struct, cu, q, stride, int(causal), scale, out, ls, ws, n), "attention_shared")
    assert M.mmshift_poll_status(ws) == status
    assert (ws[n:] == 0xA5).all()
    return out, ls


def check(got, want, what=""):
    ro, rl, tol, ltol = want
    R.check_attention(got, (ro, rl, tol + 16 * R.U32 * ro.abs().nan_to_num(0, 0, 0), ltol + 16 * R.U32), what)


def queries(new, hq, d, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((sum(new), hq, d), generator=gen, device="cuda").to(R.DT[dtype])


@pytest.mark.parametrize("dtype,kind", [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")])
@pytest.mark.parametrize("d,hq,page", [(128, 14, 16), (64, 2, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_groups(dtype, kind, d, hq, page, causal):
    groups, new = [3, 1, 4], [1, 1, 1, 2, 9, 1, 0, 3]
    lens = [[150, 170], [161, 150], [200, 133], [40, 17], [270, 300], [266, 310], [300, 290], [259, 280]]
    cache = R.Cache([lens], d, kind, page).fill_random()
    share(cache, groups, [[128 // page, 112 // page], 0, [256 // page, 17 * 16 // page]])
    q = queries(new, hq, d, dtype)
    check(attend(cache, q, new, groups, causal), R.reference(cache, q, new, causal), (dtype, kind, d, page, causal))


@pytest.mark.parametrize("common", [0, 1, 5, 8])
def test_many_rows_of_a_group(common):
    """Together the group's rows fill tiles of the tensor cores."""
    for kind in ("bf16", "i8"):
        new = [1] * 20 + [30, 2]
        cache = R.Cache([[[140 + i, 145] for i in range(22)]], 128, kind, 16).fill_random()
        share(cache, [22], [common])
        q = queries(new, 8, 128, "bf16", seed=common)
        check(attend(cache, q, new, [22]), R.reference(cache, q, new), (kind, common))


def test_what_is_common_ends_where_rows_stop_seeing_it():
    """Chunks longer than what lies behind the shared pages, sequences that end inside them, and
    sequences without rows."""
    new = [70, 3, 40, 1]
    lens = [[96], [96], [128], [0]]
    cache = R.Cache([lens], 64, "bf16", 16, room=128).fill_random()
    share(cache, [4], [6])
    q = queries(new, 4, 64, "bf16")
    for causal in (True, False):
        check(attend(cache, q, new, [4], causal), R.reference(cache, q, new, causal), causal)
    check(attend(cache, q, new, [3, 1]), R.reference(cache, q, new), "two groups")


def test_rows_longer_than_their_sequence():
    """More new rows than the sequence has: the first ones see nothing."""
    new, lens = [10, 10], [[4], [7]]
    cache = R.Cache([lens], 64, "f32", 16).fill_random()
    share(cache, [2], [1])
    q = queries(new, 2, 64, "f32")
    check(attend(cache, q, new, [2]), R.reference(cache, q, new))


@pytest.mark.parametrize("kind", ["bf16", "i8"])
def test_longer_prefix(kind):
    new = [1, 4, 1, 1, 2]
    cache = R.Cache([[[2100 + 13 * b, 1900 + b] for b in range(5)]], 128, kind, 64).fill_random(spread=2.0)
    share(cache, [5], [[30, 29]])
    q = queries(new, 14, 128, "bf16")
    check(attend(cache, q, new, [5]), R.reference(cache, q, new), kind)


@pytest.mark.parametrize("kind", ["bf16", "i8"])
def test_a_sequence_that_differs_somewhere(kind):
    """720 pages in common but for one page of one request, at the ends of what is compared at a time; requests
    without rows, and the first of a group among them."""
    new = [0, 1, 1, 0, 1, 1, 1, 2, 1, 1, 1, 1]
    for odd, at in ((1, 0), (2, 255), (4, 256), (11, 511), (10, 512), (9, 513), (5, 719), (3, 300), (0, 7)):
        cache = R.Cache([[[11520 + 3 * b, 11536 - b] for b in range(12)]], 64, kind, 16).fill_random(seed=at)
        share(cache, [12], [720])
        cache.table[0, odd, :, at] = cache.table[0, odd, :, at ^ 1]
        q = queries(new, 4, 64, "bf16", seed=at)
        for groups in ([12], [1, 11]):
            check(attend(cache, q, new, groups), R.reference(cache, q, new), (odd, at, groups))


def test_shared_pages_that_are_none():
    """Entries outside the pool, shared ones and a request's own, are left out and reported."""
    new = [1, 1, 2]
    cache = R.Cache([[[100], [90], [120]]], 64, "bf16", 16).fill_random()
    share(cache, [3], [4])
    cache.table[0, :, 0, 2] = -1
    cache.table[0, 1, 0, 5] = cache.n_pages
    q = queries(new, 4, 64, "bf16")
    table = cache.table.clone()
    gone = lambda l, b, h, pos: (table[l, b, h].long()[pos // 16] < 0) | (table[l, b, h].long()[pos // 16] >= cache.n_pages)  # noqa: E731
    check(attend(cache, q, new, [3], status=M._lib.MMSHIFT_ERR_DEVICE), R.reference(cache, q, new, gone=gone))


def test_values_that_are_not_finite():
    new = [1, 1, 40]
    cache = R.Cache([[[100], [90], [150]]], 64, "bf16", 16).fill_random()
    share(cache, [3], [4])
    for b, t, j, x in ((0, 10, 3, math.inf), (1, 70, 5, math.nan), (2, 130, 7, -math.inf), (2, 149, 9, math.nan)):
        cache.vp.view(-1, 64)[cache.slots(0, b, 0, [t])[0], j] = x
    q = queries(new, 4, 64, "bf16")
    out, lse = attend(cache, q, new, [3])
    one, lse1 = R.attend(cache, q, new)
    assert torch.equal(torch.isnan(out), torch.isnan(one)) and torch.equal(torch.isinf(out), torch.isinf(one))
    fine = torch.isfinite(one)
    assert torch.equal(out[~fine].nan_to_num(0), one[~fine].nan_to_num(0))
    # both round weights and result: two results differ by twice a bound of 2^-8 each of values below 4
    assert (out - one)[fine].abs().max() < 4 * 4 * R.UBF and (lse - lse1).abs().max() < 1e-5


def test_forked_answers_through_the_class():
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    cache = PagedKVCache(8, 2, 128, torch.bfloat16, 6, 400, page_size=32, pages=90)
    new = [200, 0, 0, 55, 0, 0]
    cache.advance(new)
    cache.append(rnd(1, 255, 2, 128), rnd(1, 255, 2, 128), new)
    cache.fork([0, 0, 3, 3], [1, 2, 4, 5])
    for new in ([1] * 6, [3, 1, 40, 0, 1, 1], [1] * 6):
        T = sum(new)
        cache.advance(new)
        cache.append(rnd(1, T, 2, 128), rnd(1, T, 2, 128), new)
        q, lse, lse1 = rnd(T, 8, 128), torch.empty((T, 8), device="cuda"), torch.empty((T, 8), device="cuda")
        a = cache.attend(q, new, groups=[3, 3], lse=lse)
        b = cache.attend(q, new, lse=lse1)
        assert (lse - lse1).abs().max() < 1e-5 and (a - b).abs().max() < 4 * 4 * R.UBF
    cache.poll()
    with pytest.raises(ValueError):
        cache.attend(q, new, groups=[3, 2])
    with pytest.raises(ValueError):
        cache.attend(q, new, groups=[6, 0])


def test_captured_and_replayed():
    """A step whose sequences grow and stop sharing between replays."""
    cache = R.Cache([[[80, 81], [90, 77], [85, 99]]], 64, "bf16", 16, room=64).fill_random()
    share(cache, [3], [4])
    new, groups = [1, 1, 1], [0, 3]
    q = queries(new, 8, 64, "bf16")
    struct = cache.struct(0)
    shape = R.shape_of(cache, new, 8, "bf16", layers=1)
    n = M.mmshift_cache_shared_workspace_size(shape, struct, groups)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.check(M.mmshift_cache_attention_shared(shape, struct, groups, q, 0, 1, 0.0, out, lse, ws, n,
                                                 torch.cuda.current_stream()), "shared")
    for step in range(3):
        graph.replay()
        check((out, lse), R.reference(cache, q, new), step)
        cache.lens.sub_(7)
        cache.lens_host = cache.lens.cpu()
        if step == 0:
            cache.table[0, 1, :, 1] = cache.table[0, 2, :, 4]     # no longer the same page
    assert M.mmshift_poll_status(ws) == M._lib.MMSHIFT_OK


def test_a_full_batch_and_strided_queries():
    new = [1 + b % 3 for b in range(64)]
    cache = R.Cache([[[150 + b, 140 + 2 * b] for b in range(64)]], 64, "bf16", 32).fill_random()
    groups = [30, 1, 33]
    share(cache, groups, [4, 0, [4, 3]])
    wide = queries(new, 10, 64, "bf16")
    q = wide[:, :6]
    for causal in (True, False):
        check(attend(cache, q, new, groups, causal, stride=wide.stride(0)), R.reference(cache, q, new, causal), causal)


def test_scales_and_no_lse():
    new = [2, 3, 1]
    cache = R.Cache([[[200], [190], [170]]], 64, "bf16", 16).fill_random()
    share(cache, [3], [9])
    q = queries(new, 40, 64, "bf16")
    check(attend(cache, q, new, [3], scale=0.3), R.reference(cache, q, new, scale=0.3))
    assert R.same(attend(cache, q, new, [3], lse=False)[0], attend(cache, q, new, [3])[0])


def test_a_first_call_is_not_captured():
    """The workspace of so many tokens would belong to the graph."""
    cache = PagedKVCache(8, 2, 64, torch.bfloat16, 2, 100, page_size=16, pages=20)
    q = queries([1, 1], 8, 64, "bf16")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError):
            cache.attend(q, [1, 1], groups=[2])
    cache.attend(q, [1, 1], groups=[2])
    cache.poll()
