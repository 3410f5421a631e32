"""Sequences that are full: rows that a call appends behind the last position are left out
and reported, and the rows that are there stay."""
import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300 import _lib as L
from paper_2607_22586_gb300.cache import PagedKVCache
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")]


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,over", [(1, 1), (1, 2), (1, 5000), (6, 1), (6, 6), (6, 7), (3, 2 ** 30 - 96), (20000, 19990)])
def test_rows_behind_a_full_sequence(dtype, kind, d, n, over):
    """96 positions; the call's rows end `over` behind them. 20,000 rows of 3 heads: the long
    call's form of the kernel."""
    cache, ref = (R.Cache([[96, 96, 50]], d, kind, 32, extra_entries=0, seed=d).fill_random() for _ in range(2))
    for c in (cache, ref):
        c.lens[0, 0] = torch.tensor([96 + over, 96, 50])
    gen = torch.Generator(device="cuda").manual_seed(n)
    K, V = (torch.randn((1, n, 3, d), generator=gen, device="cuda").to(R.DT[dtype]) for _ in range(2))
    for h, length in enumerate((96 + over, 96, 50)):
        pos = torch.arange(n) + length - n
        keep = (pos >= 0) & (pos < 96)
        if keep.any():
            ref.put(0, 0, h, pos[keep], K[0, :, h][keep.cuda()], V[0, :, h][keep.cuda()])
    shape, struct = R.shape_of(cache, [n], 3, dtype), cache.struct()
    ws, size = R.workspace(shape, struct)
    M.check(M.mmshift_cache_append(shape, struct, K, V, 0, ws, size), "append")
    assert M.mmshift_poll_status(ws) == L.MMSHIFT_ERR_DEVICE
    for got, want in zip(cache.tensors(), ref.tensors()):
        assert R.same(got, want)


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_decoding_past_the_room(dtype, kind):
    """The class: one step too many is reported by poll(), and costs no row that was there."""
    dt = R.DT[dtype]
    cache = PagedKVCache(4, 2, 64, dt, batch=1, rows=32, page_size=16, cache_dtype=R.DT[kind])
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)  # noqa: E731
    cache.advance([32])
    cache.append(rnd(1, 32, 2, 64), rnd(1, 32, 2, 64), [32])
    cache.poll()
    q, before = rnd(1, 4, 64), cache.read([32])
    want = cache.attend(q, [1])
    for step in range(3):
        cache.advance([1])
        cache.append(rnd(1, 1, 2, 64), rnd(1, 1, 2, 64), [1])
        with pytest.raises(M.MMShiftError):
            cache.poll()
        assert R.same(cache.attend(q, [1]), want)      # over the rows that the sequence holds
        for a, b in zip(cache.read([32]), before):
            assert R.same(a, b)
