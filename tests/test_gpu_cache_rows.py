"""Rows into the paged cache and back: fill, append and read against plain
indexing, to the bit; what no call writes stays as it was."""
import math

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300 import _lib as L
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")]


def _rows(shape, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=gen, device="cuda")
    # magnitudes from row to row over several decades, and a row of zeros
    x = x * torch.exp(3 * torch.randn(shape[:-1] + (1,), generator=gen, device="cuda"))
    x.view(-1, shape[-1])[0] = 0
    return x.to(R.DT[dtype])


def _check(cache, want, ws, status=0):
    assert M.mmshift_poll_status(ws) == status
    for got, ref in zip(cache.tensors(), want):
        assert R.same(got, ref)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("new,lens", [
    ([1], [[1, 40]]),
    ([3, 0, 17, 1], [[3, 5], [0, 9], [300, 17], [257, 256]]),
    ([40, 2], [[33, 40], [2, 1]]),          # longer than some sequences: the rows before their start are dropped
])
def test_append(dtype, kind, d, page, new, lens):
    cache = R.Cache([lens, lens], d, kind, page, seed=d)
    T, H = sum(new), cache.H
    K, V = _rows((2, T, H, d), dtype, 1), _rows((2, T, H, d), dtype, 2)
    ref = R.Cache([lens, lens], d, kind, page, seed=d)
    cu = R.cu_of(new)
    for l in range(2):
        for b, n in enumerate(new):
            for h in range(H):
                pos = torch.arange(n) + lens[b][h] - n
                keep = pos >= 0
                ref.put(l, b, h, pos[keep], K[l, cu[b]:cu[b + 1], h][keep.cuda()], V[l, cu[b]:cu[b + 1], h][keep.cuda()])
    shape, struct = R.shape_of(cache, new, 2 * H, dtype, stride_kv=T * H * d), cache.struct()
    ws, n = R.workspace(shape, struct)
    M.check(M.mmshift_cache_append(shape, struct, K, V, 0, ws, n), "append")
    _check(cache, ref.tensors(), ws)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("shift,pad", [(0, 8), (0, 1), (1, 0), (3, 5), (8, 16)])
def test_append_of_strided_and_unaligned_rows(dtype, kind, shift, pad):
    H, d, new, lens = 3, 64, [5, 2], [[5, 7, 30], [2, 2, 70]]
    width = (H + 2) * d + pad                          # rows inside wider ones
    buf = _rows((7 * width + 64,), dtype, 3)
    K = buf[shift:shift + 7 * width].view(7, width)[:, :H * d].unflatten(1, (H, d))
    V = buf.flip(0)[shift:shift + 7 * width].view(7, width)[:, :H * d].unflatten(1, (H, d))
    cache, ref = R.Cache(lens, d, kind, 32), R.Cache(lens, d, kind, 32)
    cu = R.cu_of(new)
    for b, n in enumerate(new):
        for h in range(H):
            ref.put(0, b, h, torch.arange(n) + lens[b][h] - n, K[cu[b]:cu[b + 1], h], V[cu[b]:cu[b + 1], h])
    shape, struct = R.shape_of(cache, new, H, dtype), cache.struct()
    ws, n = R.workspace(shape, struct)
    M.check(M.mmshift_cache_append(shape, struct, K, V, width, ws, n), "append")
    _check(cache, ref.tensors(), ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_of_special_rows(dtype):
    """Not-a-numbers, infinities, tiny and huge rows, ties between codes."""
    d = 64
    dt = R.DT[dtype]
    x = torch.zeros((12, 1, d), device="cuda")
    x[0, 0, 5] = math.nan
    x[1, 0, 6] = -math.inf
    x[2, 0, 7] = -math.nan
    x[3] = 1e-36                                       # below 2^-110
    x[4] = 2.0 ** -110
    x[5] = -3e38
    x[6] = torch.arange(d, device="cuda") + 0.5        # with a largest of 127: ties to even
    x[6, 0, -1] = 127
    x[7] = -x[6]
    x[8, 0, 63] = 1.0
    x[9] = 1e-41
    x[10] = torch.linspace(-1, 1, d, device="cuda")
    x = x.to(dt)
    cache, ref = R.Cache([[12]], d, "i8", 16), R.Cache([[12]], d, "i8", 16)
    ref.put(0, 0, 0, torch.arange(12), x[:, 0], x.flip(0)[:, 0])
    shape, struct = R.shape_of(cache, [12], 1, dtype), cache.struct()
    ws, n = R.workspace(shape, struct)
    M.check(M.mmshift_cache_append(shape, struct, x, x.flip(0), 0, ws, n), "append")
    assert M.mmshift_poll_status(ws) == 0
    for a, b in zip(cache.tensors()[:2], ref.tensors()[:2]):
        assert R.same(a, b)
    for a, b in ((cache.ks, ref.ks), (cache.vs, ref.vs)):
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and R.same(a.nan_to_num(0), b.nan_to_num(0))
    ks = cache.ks.view(-1)[cache.slots(0, 0, 0, torch.arange(12))]
    assert torch.isnan(ks[:3]).all() and torch.isfinite(ks[3:]).all()
    out = torch.empty((2, 12, 1, d), dtype=dt, device="cuda")
    M.check(M.mmshift_cache_read(shape, struct, None, out[0], out[1], ws, n), "read")
    torch.cuda.synchronize()
    assert torch.isnan(out[0, :3]).all() and torch.isfinite(out[0, 3:]).all()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("with_first", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_read(dtype, kind, d, page, with_first, shift):
    lens = [[[0, 33], [5, 5], [130, 64]], [[7, 1], [0, 0], [3, 200]]]
    rows = [40, 0, 150]
    cache = R.Cache(lens, d, kind, page).fill_random()
    T, H, dt = sum(rows), 2, R.DT[dtype]
    first = torch.tensor([[[-3, 30], [9, 9], [129, -70]], [[0, 2 ** 31 - 1], [0, 0], [-2 ** 31, 60]]],
                         dtype=torch.int32, device="cuda") if with_first else None
    want = [torch.zeros((2, T, H, d), dtype=dt, device="cuda") for _ in range(2)]
    cu = R.cu_of(rows)
    for l in range(2):
        for b, n in enumerate(rows):
            for h in range(H):
                pos = torch.arange(n) + (int(first[l, b, h]) if with_first else 0)
                ok = (pos >= 0) & (pos < lens[l][b][h])
                if ok.any():
                    at = cu[b] + torch.arange(n)[ok]
                    for w, x in zip(want, cache.get(l, b, h, pos[ok])):
                        # code * scale in float32, then the row type: float64 products are exact here
                        w[l, at.cuda(), h] = x.float().to(dt)
    shape, struct = R.shape_of(cache, rows, H, dtype), cache.struct()
    ws, n = R.workspace(shape, struct)
    buf = torch.full((2, 2 * T * H * d + 8), 7.0, dtype=dt, device="cuda")
    out = [b[shift:shift + 2 * T * H * d].view(2, T, H, d) for b in buf]
    before = cache.clone_tensors()
    M.check(M.mmshift_cache_read(shape, struct, first, *out, ws, n), "read")
    _check(cache, before, ws)
    for x, w, b in zip(out, want, buf):
        assert R.same(x.contiguous(), w)
        assert (b[:shift] == 7).all() and (b[shift + x.numel():] == 7).all()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", ["uniform", "counts"])
def test_fill(dtype, kind, d, heads):
    L_, H, page = 2, 3, 32
    seq, budgets = [300, 1, 70, 33], [50, 4, 100, 32]
    keep = [min(a, b) for a, b in zip(seq, budgets)]
    rows, T, cu, cuk = sum(keep), sum(seq), R.cu_of(seq), R.cu_of(keep)
    gen = torch.Generator().manual_seed(d)
    idx = torch.full((L_, rows, H), -1, dtype=torch.int32)
    counts = torch.zeros((L_, len(seq), H), dtype=torch.int32)
    for l in range(L_):
        for b, n in enumerate(keep):
            for h in range(H):
                c = n if heads == "uniform" else int(torch.randint(0, n + 1, (1,), generator=gen))
                counts[l, b, h] = c
                idx[l, cuk[b]:cuk[b] + c, h] = torch.randperm(seq[b], generator=gen)[:c].sort().values.to(torch.int32)
    K, V = _rows((L_, T + 5, H, d), dtype, 4), _rows((L_, T + 5, H, d), dtype, 5)    # layers further apart
    cache, ref = R.Cache(counts, d, kind, page), R.Cache(counts, d, kind, page)
    cache.lens.fill_(-77)
    for l in range(L_):
        for b in range(len(seq)):
            for h in range(H):
                c = int(counts[l, b, h])
                t = cu[b] + idx[l, cuk[b]:cuk[b] + c, h].long().cuda()
                ref.put(l, b, h, torch.arange(c), K[l, t, h], V[l, t, h])
    shape = M.make_shape(H, H, d, 2, 0 if dtype == "bf16" else 1, cu, budgets, n_layers=L_,
                         layer_stride_kv=K.stride(0), layer_stride_q=1 << 20)
    struct = cache.struct()
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    M.check(M.mmshift_cache_fill(shape, struct, K, V, idx.cuda(), None if heads == "uniform" else counts.cuda(), ws, 256),
            "fill")
    _check(cache, ref.tensors(), ws)


def test_fill_reports_bad_indices_counts_and_tables():
    H, d, page, seq = 2, 64, 16, [60]
    K, V = _rows((1, 60, H, d), "bf16", 6), _rows((1, 60, H, d), "bf16", 7)
    idx = torch.arange(40, dtype=torch.int32)[None, :, None].repeat(1, 1, H)
    shape = M.make_shape(H, H, d, 2, 0, [0, 60], [40], layer_stride_kv=0)
    for what in ("index", "count", "table", "page", "pinned"):
        cache, ref = R.Cache([[40, 40]], d, "bf16", page, extra_entries=0), R.Cache([[40, 40]], d, "bf16", page, extra_entries=0)
        i, counts, lens, status = idx.clone(), None, [40, 40], L.MMSHIFT_ERR_DEVICE
        k, v = K.clone(), V
        if what == "index":
            i[0, 3, 0], i[0, 4, 1] = 60, -1
        elif what == "count":                          # out of range: clamped
            counts, lens, status = torch.tensor([[[-4, 900]]], dtype=torch.int32, device="cuda"), [0, 40], 0
        elif what == "table":                          # two entries for three pages
            for c in (cache, ref):
                c.table = c.table[..., :2].contiguous()
            lens = [32, 32]
        elif what == "page":
            cache.table[0, 0, 1, 1] = cache.n_pages
        elif what == "pinned":                         # V in page-locked host memory, as the gather takes it
            v, status = V.cpu().pin_memory(), 0
        for h in range(H):
            n = min(lens[h], 16 if what == "page" and h == 1 else 99)
            for lo, hi in ((0, n),) if not (what == "page" and h == 1) else ((0, 16), (32, 40)):
                t = i[0, lo:hi, h].long()
                ok = (t >= 0) & (t < 60)
                x = [torch.where(ok[:, None].cuda(), y[0, t.clamp(0, 59).cuda(), h], 0) for y in (K, V)]
                ref.put(0, 0, h, torch.arange(lo, hi), *x)
        ref.table = cache.table
        ref.lens[0, 0] = torch.tensor(lens)
        struct = cache.struct()
        ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
        M.check(M.mmshift_cache_fill(shape, struct, k, v, i.cuda(), counts, ws, 256), what)
        _check(cache, ref.tensors(), ws, status)
        assert M.mmshift_poll_status(ws) == 0          # read once, cleared


def test_append_and_read_report_missing_pages():
    H, d = 1, 64
    for lens, entry in ((20, 1), (20, 0), (2 ** 31 - 1, None), (-9, None)):
        cache = R.Cache([[48]], d, "f32", 16, extra_entries=0).fill_random()
        cache.lens.fill_(lens)
        if entry is not None:
            cache.table[0, 0, 0, entry] = -1
        x = _rows((1, 6, H, d), "f32", 8)
        shape, struct = R.shape_of(cache, [6], H, "f32"), cache.struct()
        ws, n = R.workspace(shape, struct)
        before = cache.clone_tensors()
        end = min(max(lens, 0), 48)
        pos = [end - 6 + i for i in range(6)]
        ok = [p >= 0 and p // 16 != entry for p in pos]
        M.check(M.mmshift_cache_append(shape, struct, x, x, 0, ws, n), "append")
        bad = any(p >= 0 and p // 16 == entry for p in pos)
        assert M.mmshift_poll_status(ws) == (L.MMSHIFT_ERR_DEVICE if bad else 0)
        for p, o, row in zip(pos, ok, x[0, :, 0]):
            if o:
                s = cache.slots(0, 0, 0, [p])
                for a in before[:2]:
                    a.view(-1, d)[s] = row
        for a, b in zip(cache.tensors(), before):
            assert R.same(a, b)
        shape = R.shape_of(cache, [50], H, "f32")
        out = torch.empty((2, 50, d), device="cuda")
        ws, n = R.workspace(shape, struct)
        M.check(M.mmshift_cache_read(shape, struct, None, out[0], out[1], ws, n), "read")
        gone = entry is not None and entry * 16 < end
        assert M.mmshift_poll_status(ws) == (L.MMSHIFT_ERR_DEVICE if gone else 0)
        for t in range(50):
            if t < end and t // 16 != entry:
                want = cache.kp.view(-1, d)[cache.slots(0, 0, 0, [t])][0]
                assert R.same(out[0, t], want)
            else:
                assert (out[:, t] == 0).all()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_long_calls(dtype, kind, d):
    """More than 40,000 rows of all heads, of which a group of lanes takes some together: appended
    (some before a sequence's start, some not finite), read from the middle on, and filled."""
    H, new, lens = 3, [9001, 0, 5003], [[9001, 9500, 8000], [4, 5, 6], [5003, 1, 5100]]
    T, cu = sum(new), R.cu_of(new)
    K, V = _rows((1, T, H, d), dtype, 1), _rows((1, T, H, d), dtype, 2)
    K[0, 70, :, 3] = math.inf
    V[0, 71, 1, 5] = math.nan
    cache, ref = R.Cache(lens, d, kind, 64, seed=d), R.Cache(lens, d, kind, 64, seed=d)
    for b, n in enumerate(new):
        for h in range(H):
            pos = torch.arange(n) + lens[b][h] - n
            keep = pos >= 0
            ref.put(0, b, h, pos[keep], K[0, cu[b]:cu[b + 1], h][keep.cuda()], V[0, cu[b]:cu[b + 1], h][keep.cuda()])
    shape, struct = R.shape_of(cache, new, 2 * H, dtype), cache.struct()
    ws, n = R.workspace(shape, struct)
    M.check(M.mmshift_cache_append(shape, struct, K, V, 0, ws, n), "append")

    def check():
        assert M.mmshift_poll_status(ws) == 0
        for got, want in zip(cache.tensors(), ref.tensors()):
            if got.is_floating_point():
                assert torch.equal(torch.isnan(got), torch.isnan(want))
                got, want = got.nan_to_num(0, 1, -1), want.nan_to_num(0, 1, -1)
            assert R.same(got, want)

    check()
    first = torch.tensor([[[0, 400, 7999], [0, 0, 0], [3, 0, 100]]], dtype=torch.int32)
    out = torch.full((2, T, H, d), 9.0, dtype=R.DT[dtype], device="cuda")
    M.check(M.mmshift_cache_read(shape, struct, first.cuda(), out[0], out[1], ws, n), "read")
    assert M.mmshift_poll_status(ws) == 0
    for b, m in enumerate(new):
        for h in range(H):
            pos = torch.arange(m) + int(first[0, b, h])
            pos = pos[pos < lens[b][h]]
            want = cache.get(0, b, h, pos)
            for x, w in zip(out[:, cu[b]:cu[b + 1], h], want):
                w = w.float().to(R.DT[dtype])
                assert torch.equal(torch.isnan(x[:len(pos)]), torch.isnan(w))
                assert R.same(x[:len(pos)].nan_to_num(0, 1, -1).contiguous(), w.nan_to_num(0, 1, -1))
                assert (x[len(pos):] == 0).all()

    seq, budgets = [9001, 1, 5003], [8000, 1, 5003]
    keep = [min(a, b) for a, b in zip(seq, budgets)]
    K, V = _rows((1, sum(seq), H, d), dtype, 3), _rows((1, sum(seq), H, d), dtype, 4)
    cache, ref = (R.Cache([[n] * H for n in keep], d, kind, 64, seed=1) for _ in range(2))
    cache.lens.fill_(-77)
    gen, at, cuk = torch.Generator().manual_seed(6), R.cu_of(seq), R.cu_of(keep)
    idx = torch.zeros((1, sum(keep), H), dtype=torch.int32)
    for b, m in enumerate(keep):
        for h in range(H):
            t = torch.randperm(seq[b], generator=gen)[:m].sort().values
            idx[0, cuk[b]:cuk[b + 1], h] = t.int()
            ref.put(0, b, h, torch.arange(m), K[0, at[b] + t.cuda(), h], V[0, at[b] + t.cuda(), h])
    shape, struct = M.make_shape(H, H, d, 2, 0 if dtype == "bf16" else 1, at, budgets), cache.struct()
    M.check(M.mmshift_cache_fill(shape, struct, K, V, idx.cuda(), None, ws, 256), "fill")
    check()
