"""PagedKVCache: a selection's rows, a chunk and single tokens through the class,
against attention over dense copies of the same rows; its refusals; captured steps."""
import math

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300.cache import PagedKVCache
from paper_2607_22586_gb300.selector import KVSelector
from tests import cache_ref as R


def _cache(**kw):
    a = dict(n_q_heads=6, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, batch=2, rows=100, n_layers=2, page_size=16)
    a.update(kw)
    return PagedKVCache(**a)


def _view(cache):
    """The class's cache as the tests' reference reads one."""
    v = R.Cache.__new__(R.Cache)
    v.L, v.B, v.H = cache.lens.shape
    v.d, v.page, v.n_pages = cache.head_dim, cache.k_pages.shape[1], len(cache.k_pages)
    v.kind = {torch.int8: "i8", torch.bfloat16: "bf16", torch.float32: "f32"}[cache.cache_dtype]
    v.table, v.lens, v.lens_host = cache.page_table, cache.lens, cache.lens.cpu()
    v.kp, v.vp, v.ks, v.vs = cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales
    return v


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind", [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")])
@pytest.mark.parametrize("head_budgets", [False, True])
def test_selection_chunk_and_tokens(dtype, kind, head_budgets):
    dt = R.DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)  # noqa: E731
    seq, budgets = [200, 90], [50, 30]
    sel = KVSelector(6, 2, 64, 8, dt, R.cu_of(seq), budgets, n_layers=2, params=M.default_params(n_proxies=32, n_groups=2))
    K, V, Q = rnd(2, 290, 2, 64), rnd(2, 290, 2, 64), rnd(2, 2, 8, 6, 64)
    hb = torch.randint(1, 30, (2, 2, 2), generator=gen, device="cuda", dtype=torch.int32) if head_budgets else None
    idx, kk, vv = sel(K, V, Q, head_budgets=hb)
    cache = _cache(dtype=dt, cache_dtype=R.DT[kind])
    cache.fill(sel, K, V)
    kept = sel.out_count if head_budgets else torch.tensor(budgets, device="cuda")[None, :, None].expand(2, 2, 2)
    assert torch.equal(cache.lens, kept.int())
    k, v = cache.read(budgets)
    for got, want in ((k, kk), (v, vv)):
        if kind == "i8":
            code, scale = R.quantise(want)
            want = (code.float() * scale[..., None]).to(dt)
        assert R.same(got, want)
    for new in ([20, 1], [1, 1], [1, 0]):
        T = sum(new)
        qkv = rnd(2, T, 10 * 64)                            # one projection's output
        q, k, v = (x.unflatten(-1, (-1, 64)) for x in qkv.split([6 * 64, 2 * 64, 2 * 64], -1))
        cache.advance(new)
        cache.append(k, v, new)
        for layer in range(2):
            lse = torch.empty((T, 6), device="cuda")
            out = cache.attend(q[layer], new, layer, lse=lse)
            R.check_attention((out, lse), R.reference(_view(cache), q[layer], new, layer=layer))
    cache.poll()


@pytest.mark.gpu
def test_captured_steps_of_two_batches():
    """Two captured steps with row counts of their own, replayed in turn."""
    cache = _cache(rows=torch.randint(60, 100, (2, 2, 2)))
    gen = torch.Generator(device="cuda").manual_seed(3)
    steps = []
    for new in ([1, 1], [3, 2]):
        T = sum(new)
        q, k, v = (torch.zeros((2, T, h, 64), dtype=torch.bfloat16, device="cuda") for h in (6, 2, 2))
        out = torch.zeros_like(q)
        cache.advance(new)                                  # once outside a capture: workspaces made
        cache.append(k, v, new)
        cache.attend(q[0], new, 0, out=out[0])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.advance(new)
            cache.append(k, v, new)
            for layer in range(2):
                cache.attend(q[layer], new, layer, out=out[layer])
        steps.append((new, q, k, v, out, g))
    cache.lens.zero_()
    for i in range(12):
        new, q, k, v, out, g = steps[i % 2]
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        g.replay()
        cache.poll()
        for layer in range(2):
            want = R.reference(_view(cache), q[layer], new, layer=layer)
            R.check_attention((out[layer], want[1].float()), (want[0], want[1], want[2], want[3] + 1e-3))


@pytest.mark.gpu
def test_another_stream_and_one_layer_at_a_time():
    cache, ref = _cache(), _cache()
    s = torch.cuda.Stream()
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn((2, 9, 2, 64), generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((9, 6, 64), generator=gen, device="cuda").bfloat16()
    new = [4, 5]
    ref.advance(new)
    ref.append(k, v, new)
    want = ref.attend(q, new, 1, causal=False, softmax_scale=0.2)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        cache.advance(new)
        for layer in (1, 0):
            cache.append(k[layer], v[layer], new, layer)
        out = cache.attend(q, new, 1, causal=False, softmax_scale=0.2)
        cache.poll()
    torch.cuda.synchronize()
    assert R.same(out, want)
    for a, b in ((cache.k_pages, ref.k_pages), (cache.v_pages, ref.v_pages)):
        assert R.same(a, b)


@pytest.mark.gpu
def test_refusals():
    cache = _cache()
    q, k = torch.zeros((3, 6, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: cache.attend(q, [1, 1]), lambda: cache.attend(q, [3]), lambda: cache.attend(q.float(), [1, 2]),
                 lambda: cache.attend(q.transpose(0, 1), [1, 2]), lambda: cache.attend(q.cpu(), [1, 2]),
                 lambda: cache.attend(q, [1, 2], out=q[:2]), lambda: cache.attend(q, [1, 2], lse=torch.zeros(3, 6)),
                 lambda: cache.append(k, k[0], [1, 2]), lambda: cache.append(k[0], k[0], [1, 2]),
                 lambda: cache.append(k, k[..., ::2], [1, 2]), lambda: cache.advance([1]),
                 lambda: cache.read([1, 2], torch.zeros(2, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(M.MMShiftError):
        cache.attend(q, [1, 2], softmax_scale=math.nan)
    with pytest.raises(IndexError):
        cache.attend(q, [1, 2], layer=2)


def test_constructor_refusals():
    for bad in (dict(dtype=torch.float16), dict(cache_dtype=torch.float32), dict(rows=0), dict(rows=[[[1, 0], [1, 1]]] * 2)):
        with pytest.raises(ValueError):
            _cache(device="cpu", **bad)
    c = _cache(device="cpu", rows=[[[1, 16], [17, 40]], [[3, 3], [100, 1]]])
    assert c.page_table.shape == (2, 2, 2, 7) and c.capacity == 16
    used = c.page_table[c.page_table >= 0]
    assert sorted(used.tolist()) == list(range(1 + 1 + 2 + 3 + 1 + 1 + 7 + 1)) and len(c.k_pages) == 17
    assert c.page_table[1, 1, 0].tolist() == list(range(9, 16)) and c.page_table[0, 0, 0].tolist() == [0] + [-1] * 6


def test_rows_that_overlap_or_have_other_axes_are_refused():
    """Before anything is launched: without a GPU."""
    c = _cache(device="cpu")
    q, k = torch.zeros((1, 6, 64), dtype=torch.bfloat16), torch.zeros((2, 1, 2, 64), dtype=torch.bfloat16)
    flat = torch.zeros(3 * 384, dtype=torch.bfloat16)
    for call in (lambda: c.attend(q.expand(3, 6, 64), [1, 2]),                       # one row for all tokens
                 lambda: c.attend(flat.as_strided((3, 6, 64), (320, 64, 1)), [1, 2]),
                 lambda: c.append(k.expand(2, 3, 2, 64), k.expand(2, 3, 2, 64), [1, 2]),
                 lambda: c.attend(torch.zeros((2, 3, 6, 64), dtype=torch.bfloat16), [1, 2]),
                 lambda: c.append(k.expand(2, 1, 2, 64), k, [1, 0], layer=1)):
        with pytest.raises(ValueError):
            call()


def test_indices_of_another_shape_or_type_are_refused():
    """Before anything is launched: without a GPU."""
    c, sel = _cache(device="cpu", batch=1), KVSelector.__new__(KVSelector)
    sel.__dict__.update(n_layers=2, budgets=[5], n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, device=c.device,
                        out_idx=torch.zeros((2, 5, 2), dtype=torch.int32), out_count=None, _check=lambda *a: None)
    k = torch.zeros((2, 9, 2, 64), dtype=torch.bfloat16)
    idx, counts = sel.out_idx, torch.zeros((2, 1, 2), dtype=torch.int32)
    for i, n in ((idx.long(), None), (idx[:, :4], None), (idx.transpose(0, 2), None), (idx, counts.long()),
                 (idx, counts[:1])):
        with pytest.raises(ValueError):
            c.fill(sel, k, k, i, n)


@pytest.mark.parametrize("dtype,kind", [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")])
def test_the_workspace_does_for_every_call(dtype, kind):
    """And what is kept for combinations of row counts does not grow without end."""
    g = torch.Generator().manual_seed(11)
    for r in (1, 3, 7, 9, 11, 16, 17, 31, 32, 33, 64, 65, 300):
        for batch in (1, 3):
            c = _cache(device="cpu", n_q_heads=2 * r, dtype=R.DT[dtype], batch=batch, head_dim=128 if r % 2 else 64,
                       cache_dtype=torch.int8 if kind == "i8" else None)
            calls = [[n] * batch for n in range(1, 70)] + [[n] + [1] * (batch - 1) for n in (256, 300, 1000)]
            calls += [(2 ** torch.randint(0, 13, (batch,), generator=g)).tolist() for _ in range(40)]
            assert max(c._shape(new, 1)[1] for new in calls) <= c._ws_bytes
    for n in range(1000):
        c._call([n, 1, 2], 1)
        c.advance([n, 1, 2])
    assert len(c._calls) <= 256 and len(c._counts) <= 256 and not c._captured
