"""Attention over the paged cache against the formula in float64, element by element
within a bound that counts the roundings (cache_ref.reference)."""
import math

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300 import _lib as L
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")]


def _q(new, hq, d, dtype, seed=3, spread=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (spread * torch.randn((sum(new), hq, d), generator=gen, device="cuda")).to(R.DT[dtype])


def _run(lens, new, hq, d, dtype, kind, page, causal=True, seed=0, spread=1.0, scale=0.0):
    cache = R.Cache(lens, d, kind, page, seed=seed).fill_random(seed + 1, spread)
    q = _q(new, hq, d, dtype, seed + 2)
    before = cache.clone_tensors()
    got = R.attend(cache, q, new, causal, scale)
    R.check_attention(got, R.reference(cache, q, new, causal, scale))
    for a, b in zip(cache.tensors(), before):
        assert R.same(a, b)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[[1]], [[15]], [[16]], [[17]], [[63]], [[64]], [[129]], [[700]]])
def test_one_token_one_head(dtype, kind, d, lens):
    _run(lens, [1], 1, d, dtype, kind, 16)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_tokens_of_a_batch(dtype, kind, d, page):
    """One token each, heads of different lengths, one sequence empty."""
    _run([[1, 40], [300, 0], [257, 256], [5, 1111]], [1, 1, 1, 1], 14, d, dtype, kind, page, seed=page)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("r", [1, 2, 3, 7, 8, 16])
@pytest.mark.parametrize("n", [1, 2, 5])
def test_group_sizes(dtype, kind, d, r, n):
    _run([[n + 37, n], [200, n + 250]], [n, n], 2 * r, d, dtype, kind, 32, seed=r)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new,lens", [
    ([33], [[33, 40]]),
    ([129, 1], [[129, 500], [64, 1]]),
    ([1, 0, 70, 18, 2], [[130, 1], [9, 9], [70, 333], [18, 300], [2, 2]]),
    ([40, 3], [[0, 17], [3, 2]]),                      # sequences shorter than the chunk: rows without keys
    ([37, 260], [[600, 37], [260, 700]]),
])
def test_chunks(dtype, kind, d, causal, new, lens):
    _run(lens, new, 6, d, dtype, kind, 16, causal, seed=len(new))


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_many_heads_and_requests(dtype, kind):
    B = 64
    lens = [[1 + (37 * b + 11 * h) % 90 for h in range(3)] for b in range(B)]
    new = [1 + (b % 3 == 0) * (b % 5) for b in range(B)]
    _run(lens, new, 9, 64, dtype, kind, 16)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("n", [1, 24])
def test_long_sequence(dtype, kind, n):
    _run([[9001]], [n], 2, 128, dtype, kind, 64)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_long_chunk(dtype, kind, d):
    """Several row tiles, rings of tiles gone round many times."""
    _run([[4500, 300]], [150], 6, d, dtype, kind, 32)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("n,r", [(1, 2), (2, 9)])
def test_more_sequences_than_any_list_holds(dtype, kind, n, r):
    """1,088 and 2,816 sequences of a few rows: lengths that do not fit in shared memory, workers
    with more units than are listed ahead."""
    B, H = 64, 17 if n == 1 else 44
    lens = [[(5 * b + 7 * h) % 23 for h in range(H)] for b in range(B)]
    _run(lens, [n] * B, H * r, 64, dtype, kind, 16)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("n", [1, 20])
def test_large_logits_and_scale(dtype, kind, n):
    """Logits of hundreds, the largest anywhere: the running maximum has to follow."""
    _run([[800, 333]], [n], 4, 64, dtype, kind, 16, spread=30.0)
    _run([[800, 333]], [n], 4, 64, dtype, kind, 16, scale=2.5)


def _special(dtype, kind, n, edit, lens=150, hq=4, d=64, causal=True, gone=None, status=0, new=None, seed=0):
    cache = R.Cache([[lens, lens + 9]], d, kind, 16, seed=seed).fill_random(5)
    new = new or [n]
    q = _q(new, hq, d, dtype)
    edit(cache, q)
    got = R.attend(cache, q, new, causal, status=status)
    R.check_attention(got, R.reference(cache, q, new, causal, gone=gone))
    return got


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("n", [1, 2, 3, 40])
@pytest.mark.parametrize("what", ["nan", "inf"])
@pytest.mark.parametrize("side", ["k", "v"])
def test_not_finite_rows_reach_only_their_own_readers(dtype, kind, n, what, side):
    """The last token's own row is not finite: the tokens before it do not attend to it. (An 8-bit
    row with an infinity reads as NaN.)"""
    bad = math.nan if what == "nan" else math.inf

    def edit(cache, q):
        for h in range(2):
            x = [torch.randn((1, 64), device="cuda") for _ in range(2)]
            x["kv".index(side)][0, 7] = bad
            cache.put(0, 0, h, [int(cache.lens_host[0, 0, h]) - 1], *x)

    out, _ = _special(dtype, kind, n, edit)
    assert not torch.isfinite(out[-1]).all()
    assert torch.isfinite(out[:-1]).all()


@pytest.mark.parametrize("dtype,kind", [k for k in KINDS if k[1] != "i8"])
@pytest.mark.parametrize("n", [1, 3, 40])
def test_infinite_logits(dtype, kind, n):
    """Keys with z = -inf count for nothing; a token whose keys all have it gets what one without
    keys gets; z = +inf makes a NaN."""
    def minus(cache, q):
        q[..., 0] = q[..., 0].abs() + 0.1
        k, v = cache.get(0, 0, 0, torch.arange(150))
        k[20:90, 0] = -math.inf
        cache.put(0, 0, 0, torch.arange(150), k, v)

    _special(dtype, kind, n, minus)

    def every(cache, q):
        q[..., 0] = q[..., 0].abs() + 0.1
        k, v = cache.get(0, 0, 0, torch.arange(150))
        k[:, 0] = -math.inf
        cache.put(0, 0, 0, torch.arange(150), k, v)

    cache = R.Cache([[150, 159]], 64, kind, 16).fill_random(5)
    q = _q([n], 4, 64, dtype)
    every(cache, q)
    out, lse = R.attend(cache, q, [n])
    assert (out[:, :2] == 0).all() and (lse[:, :2] == -math.inf).all()
    assert torch.isfinite(out[:, 2:]).all() and torch.isfinite(lse[:, 2:]).all()

    def plus(cache, q):
        q[..., 0] = q[..., 0].abs() + 0.1
        k, v = cache.get(0, 0, 0, [100])
        k[0, 0] = math.inf
        cache.put(0, 0, 0, [100], k, v)

    cache = R.Cache([[150, 159]], 64, kind, 16).fill_random(5)
    plus(cache, q)
    out, _ = R.attend(cache, q, [n])
    assert torch.isnan(out[:, :2]).all() and torch.isfinite(out[:, 2:]).all()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("n", [1, 6, 50])
@pytest.mark.parametrize("entries", [[0], [3], [9], [1, 2, 3, 4, 5, 6, 7, 8], list(range(10))])
def test_missing_pages_are_left_out(dtype, kind, n, entries):
    def edit(cache, q):
        cache.table[0, 0, 0, entries] = torch.tensor([-1, cache.n_pages, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32,
                                                     device="cuda").repeat(3)[:len(entries)]

    def gone(l, b, h, pos):
        return torch.isin(pos // 16, torch.tensor(entries, device="cuda")) & (h == 0)

    cache = R.Cache([[150, 159]], 64, kind, 16).fill_random(5)
    q = _q([n], 4, 64, dtype)
    want = cache.table.clone()
    ref = None
    # the reference reads the table before it is spoiled
    ref = R.reference(cache, q, [n], gone=gone)
    edit(cache, q)
    R.check_attention(R.attend(cache, q, [n], status=L.MMSHIFT_ERR_DEVICE), ref)
    cache.table.copy_(want)
    R.check_attention(R.attend(cache, q, [n]), R.reference(cache, q, [n]))


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("n", [1, 30])
def test_lengths_outside_the_table_are_clamped(dtype, kind, n):
    cache = R.Cache([[160, 160]], 64, kind, 16, extra_entries=0).fill_random(5)
    q = _q([n], 4, 64, dtype)
    want = R.attend(cache, q, [n])
    cache.lens.copy_(torch.tensor([[[161, 2 ** 31 - 1]]]))
    got = R.attend(cache, q, [n])
    assert R.same(got[0], want[0]) and R.same(got[1], want[1])
    cache.lens.copy_(torch.tensor([[[-1, -2 ** 31]]]))
    out, lse = R.attend(cache, q, [n])
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("n", [1, 4, 40])
@pytest.mark.parametrize("shift,pad,oshift", [(0, 8, 0), (1, 0, 0), (0, 1, 1), (3, 3, 5)])
def test_strided_and_unaligned_rows(dtype, kind, n, shift, pad, oshift):
    d, hq, new = 64, 6, [n, 2]
    cache = R.Cache([[90, 45], [2, 33]], d, kind, 32).fill_random()
    T, width = sum(new), hq * d + 4 * d + pad
    buf = _q([T * width + 64], 1, 1, dtype).view(-1)
    q = buf[shift:shift + T * width].view(T, width)[:, :hq * d].unflatten(1, (hq, d))
    room = torch.full((T * hq * d + 64,), 7.0, dtype=q.dtype, device="cuda")
    out = room[oshift:oshift + T * hq * d].view(T, hq, d)
    got = R.attend(cache, q, new, stride=width, out=out)
    R.check_attention(got, R.reference(cache, q, new))
    assert (room[:oshift] == 7).all() and (room[oshift + out.numel():] == 7).all()
    assert R.same(out.contiguous(), R.attend(cache, q.contiguous(), new, lse=False)[0])


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_same_bits_every_time(dtype, kind):
    new = [1, 30, 3, 1]
    cache = R.Cache([[900, 70], [500, 31], [3, 260], [0, 1]], 128, kind, 16).fill_random()
    q = _q(new, 14, 128, dtype)
    a = R.attend(cache, q, new)
    for _ in range(3):
        b = R.attend(cache, q, new)
        assert R.same(a[0], b[0]) and R.same(a[1], b[1])


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_shared_pages(dtype, kind):
    """Two sequences whose first pages are the same ones (a common prefix)."""
    cache = R.Cache([[100], [80]], 64, kind, 16).fill_random()
    cache.table[0, 1, 0, :4] = cache.table[0, 0, 0, :4]
    q = _q([2, 30], 3, 64, dtype)
    R.check_attention(R.attend(cache, q, [2, 30]), R.reference(cache, q, [2, 30]))


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_a_captured_step_follows_the_sequences(dtype, kind):
    """append + attention captured once, replayed while lens grows; two graphs share a workspace."""
    B, H, hq, d, steps = 3, 2, 6, 64, 20
    start = [[5, 30], [16, 0], [100, 47]]
    cache = R.Cache(start, d, kind, 16, room=steps).fill_random()
    dt = R.DT[dtype]
    q, k, v = (torch.zeros((B, n, d), dtype=dt, device="cuda") for n in (hq, H, H))
    shape, struct = R.shape_of(cache, [1] * B, hq, dtype), cache.struct()
    ws, n = R.workspace(shape, struct)
    outs = [torch.zeros((B, hq, d), dtype=dt, device="cuda") for _ in range(2)]
    lse = torch.zeros((B, hq), device="cuda")
    graphs = []
    for out in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s = torch.cuda.current_stream()
            cache.lens.add_(1)
            M.check(M.mmshift_cache_append(shape, struct, k, v, 0, ws, n, s), "append")
            M.check(M.mmshift_cache_attention(shape, struct, q, 0, 1, 0.0, out, lse, ws, n, s), "attention")
        graphs.append(g)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for step in range(steps):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        graphs[step % 2].replay()
        assert M.mmshift_poll_status(ws) == 0
        cache.lens_host = cache.lens.cpu()
        assert cache.lens_host.flatten().tolist() == [x + step + 1 for row in start for x in row]
        R.check_attention((outs[step % 2], lse), R.reference(cache, q, [1] * B), step)


def test_two_streams_at_once():
    new = [1, 40]
    caches = [R.Cache([[700, 70], [500, 41]], 128, "i8", 16, seed=s).fill_random(s) for s in range(2)]
    qs = [_q(new, 14, 128, "bf16", s) for s in range(2)]
    want = [R.attend(c, q, new) for c, q in zip(caches, qs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    shape, structs = R.shape_of(caches[0], new, 14, "bf16"), [c.struct() for c in caches]
    spaces = [R.workspace(shape, s) for s in structs]
    outs = [torch.zeros_like(q) for q in qs]
    lses = [torch.zeros(q.shape[:2], device="cuda") for q in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            M.check(M.mmshift_cache_attention(shape, structs[i], qs[i], 0, 1, 0.0, outs[i], lses[i], *spaces[i], streams[i]), "a")
    for i in range(2):
        assert M.mmshift_poll_status(spaces[i][0], streams[i]) == 0
        assert R.same(outs[i], want[i][0]) and R.same(lses[i], want[i][1])


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("head_budgets", [False, True])
def test_selection_then_decoding(dtype, kind, head_budgets):
    """The whole path: a selection, its kept rows into the cache, a chunk and a token appended and
    attended to, against attention over the kept rows and the new ones."""
    L_, hq, H, d, W = 2, 14, 2, 128, 8
    seq, budgets = [260, 130], [60, 40]
    dt = R.DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)  # noqa: E731
    cu = R.cu_of(seq)
    from paper_2607_22586_gb300.selector import KVSelector
    sel = KVSelector(hq, H, d, W, dt, cu, budgets, n_layers=L_, params=M.default_params(n_proxies=32, n_groups=2))
    K, V, Q = rnd(L_, cu[-1], H, d), rnd(L_, cu[-1], H, d), rnd(L_, 2, W, hq, d)
    hb = torch.randint(1, 40, (L_, 2, H), generator=gen, device="cuda", dtype=torch.int32) if head_budgets else None
    idx, kk, vv = sel(K, V, Q, head_budgets=hb)
    counts = sel.out_count if head_budgets else torch.tensor(budgets, dtype=torch.int32, device="cuda")[None, :, None].expand(L_, 2, H).contiguous()
    cache = R.Cache(counts.cpu(), d, kind, 16, room=20)
    cache.lens.zero_()
    ws, n = R.workspace(R.shape_of(cache, [9, 9], hq, dtype), cache.struct())
    M.check(M.mmshift_cache_fill(sel.shape, cache.struct(), K, V, idx, counts if head_budgets else None, ws, n), "fill")
    assert torch.equal(cache.lens, counts)
    rows = [min(a, b) for a, b in zip(seq, budgets)]
    out = [torch.zeros_like(kk) for _ in range(2)]
    M.check(M.mmshift_cache_read(R.shape_of(cache, rows, hq, dtype), cache.struct(), None, *out, ws, n), "read")
    for got, kept in zip(out, (kk, vv)):               # the gather's rows, as the cache holds them
        if kind == "i8":
            code, scale = R.quantise(kept)
            kept = (code.float() * scale[..., None]).to(dt)
        assert R.same(got, kept)
    for new in ([7, 5], [1, 1]):
        cache.lens.add_(torch.tensor(new, dtype=torch.int32, device="cuda")[None, :, None])
        cache.lens_host = cache.lens.cpu()
        k, v, q = rnd(L_, sum(new), H, d), rnd(L_, sum(new), H, d), rnd(L_, sum(new), hq, d)
        shape = R.shape_of(cache, new, hq, dtype, stride_kv=k.stride(0))
        M.check(M.mmshift_cache_append(shape, cache.struct(), k, v, 0, ws, n), "append")
        for layer in range(L_):
            R.check_attention(R.attend(cache, q[layer], new, layer=layer), R.reference(cache, q[layer], new, layer=layer))
    assert M.mmshift_poll_status(ws) == 0


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_pages_past_32_bits_of_bytes(dtype, kind):
    """The same pages behind the first 4 GB of a pool: same bits written, read and attended to."""
    d, new, hq = 128, [1, 40, 100], 6
    small = R.Cache([[300, 1], [90, 41], [700, 100]], d, kind, 64).fill_random()
    row = d * small.kp.element_size()
    shift = 2 ** 32 // (row * 64) + 5
    big = R.Cache.__new__(R.Cache)
    big.__dict__.update(small.__dict__, n_pages=shift + small.n_pages)
    big.table = torch.where((small.table >= 0) & (small.table < small.n_pages), small.table + shift, -1).int()
    for name in ("kp", "vp", "ks", "vs"):
        pages = getattr(small, name)
        if pages is not None:
            far = torch.empty((big.n_pages, *pages.shape[1:]), dtype=pages.dtype, device="cuda")
            far[shift:] = pages
            setattr(big, name, far)
    q = _q(new, hq, d, dtype)
    gen = torch.Generator(device="cuda").manual_seed(8)
    k, v = (torch.randn((sum(new), 2, d), generator=gen, device="cuda").to(R.DT[dtype]) for _ in range(2))
    shape, got = R.shape_of(small, new, hq, dtype), []
    for c in (small, big):
        struct = c.struct()
        ws, n = R.workspace(shape, struct)
        s = torch.cuda.current_stream()
        M.check(M.mmshift_cache_append(shape, struct, k, v, 0, ws, n, s), "append")
        out = [torch.empty_like(q)] + [torch.empty((sum(new), 2, d), dtype=R.DT[dtype], device="cuda") for _ in range(2)]
        lse = torch.empty(q.shape[:2], device="cuda")
        M.check(M.mmshift_cache_read(shape, struct, None, out[1], out[2], ws, n, s), "read")
        M.check(M.mmshift_cache_attention(shape, struct, q, 0, 1, 0.0, out[0], lse, ws, n, s), "attention")
        assert M.mmshift_poll_status(ws) == 0
        got.append(out + [lse] + [t[-small.n_pages:] for t in (c.kp, c.vp, c.ks, c.vs) if t is not None])
    for a, b in zip(*got):
        assert R.same(a, b)
