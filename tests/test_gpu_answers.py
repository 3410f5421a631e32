"""One prompt, many answers: rotation, attention over the prompt, selection, pages, forks, drafts and
single tokens over shared pages, compaction and release, as a serving program has them in a
row, against dense rows in float64."""
import math

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300.cache import PagedKVCache
from paper_2607_22586_gb300.prompt import PromptAttention, Rotary
from paper_2607_22586_gb300.selector import KVSelector
from tests import cache_ref as R
from tests import test_gpu_prompt, test_gpu_rope

pytestmark = pytest.mark.gpu

HQ, HKV, L, W = 8, 2, 2, 8


def dense(q, keys, values, n):
    """Attention of the last n tokens' queries [n, r, d] over a sequence's rows, with its tolerances."""
    r, d, m = q.shape[1], q.shape[2], len(keys)
    z = torch.einsum("nrd,md->rnm", q.double(), keys) / math.sqrt(d)
    seen = torch.arange(m, device="cuda") <= torch.arange(m - n, m, device="cuda")[:, None]
    z = z.masked_fill(~seen, -math.inf)
    p = torch.softmax(z, -1)
    zerr = (d + 4) * R.U32 * (torch.einsum("nrd,md->rnm", q.double().abs(), keys.abs()) / math.sqrt(d)).amax(-1, keepdim=True)
    out = torch.einsum("rnm,md->nrd", p, values)
    rel = (4 * zerr + (32 + 2 * m) * R.U32 + R.UBF + R.U32).transpose(0, 1)
    return out, 1.01 * (rel * torch.einsum("rnm,md->nrd", p, values.abs()) + R.UBF * out.abs()) + 1e-37


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("d", [64, 128])
def test_one_prompt_many_answers(kind, d):
    gen = torch.Generator(device="cuda").manual_seed(d)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    T, budget, batch = 300, 90, 5
    rotary = Rotary(d, theta=1e5, sections=(d // 8, d // 8, d // 4))
    attention = PromptAttention(HQ, HKV, d, torch.bfloat16, [0, T])
    pos = torch.randint(0, T, (3, T), generator=gen, device="cuda", dtype=torch.int32)
    raw_q, raw_k, V = rnd(L, T, HQ, d), rnd(L, T, HKV, d), rnd(L, T, HKV, d)
    Q, K = rotary(raw_q, raw_k, pos)
    args = (pos, rotary.inv_freq, "half", rotary.sections, 1.0)
    test_gpu_rope.check(Q, raw_q, *args)
    test_gpu_rope.check(K, raw_k, *args)
    for layer in range(L):
        lse = torch.empty((T, HQ), device="cuda")
        out = attention(Q[layer], K[layer], V[layer], lse=lse)
        R.check_attention((out, lse), test_gpu_prompt.reference(Q[layer], K[layer], V[layer], [0, T], True))
    sel = KVSelector(HQ, HKV, d, W, torch.bfloat16, [0, T], [budget], n_layers=L,
                     params=M.default_params(n_proxies=32, n_groups=2))
    idx, kk, vv = sel(K, V, Q[:, -W:].transpose(0, 0).contiguous().view(L, 1, W, HQ, d))
    cache = PagedKVCache(HQ, HKV, d, torch.bfloat16, batch, 256, n_layers=L, page_size=16,
                         cache_dtype=R.DT[kind], pages=L * batch * HKV * 16)
    # the kept rows as the first request's, then four answers to it
    cache.advance([budget] + [0] * 4)
    cache.append(kk, vv, [budget] + [0] * 4)
    cache.fork([0] * 4, [1, 2, 3, 4])
    held = cache.refs.clone()
    assert int(held.max()) == batch

    def as_held(x):
        if kind != "i8":
            return x.double()
        code, scale = R.quantise(x)
        return code.double() * scale.double()[..., None]

    rows = [[[[as_held(x[l, :, h]) for x in (kk, vv)] for h in range(HKV)] for _ in range(batch)] for l in range(L)]
    for step, new in enumerate(([1] * 5, [3, 1, 4, 1, 2], [1] * 5, [40, 0, 1, 1, 1])):
        n = sum(new)
        cu = R.cu_of(new)
        p = (T + step * 8 + torch.arange(n, device="cuda")).to(torch.int32).expand(3, n).contiguous()
        q, k = rotary(rnd(L, n, HQ, d), rnd(L, n, HKV, d), p)
        v = rnd(L, n, HKV, d)
        cache.advance(new)
        cache.append(k, v, new)
        for l in range(L):
            out = cache.attend(q[l], new, l, groups=[5] if step % 2 else [2, 3])
            for b in range(batch):
                for h in range(HKV):
                    now = rows[l][b][h]
                    for i, x in enumerate((k, v)):
                        now[i] = torch.cat([now[i], as_held(x[l, cu[b]:cu[b + 1], h])])
                    if new[b]:
                        want, tol = dense(q[l, cu[b]:cu[b + 1], h * 4:(h + 1) * 4], *now, new[b])
                        got = out[cu[b]:cu[b + 1], h * 4:(h + 1) * 4].double()
                        assert ((got - want).abs() <= tol).all(), (step, l, b, h)
    # two answers keep every other row, one is done. The second has 93 rows, so that the last of its 48
    # indices, 94, is none of them: a zero row, which is reported
    counts = [0, 48, 0, 47, 0]
    idx = torch.cat([torch.arange(0, 2 * c, 2) for c in counts]).to(torch.int32)[None, :, None]
    cache.compact(idx.expand(L, sum(counts), HKV).contiguous().cuda(), counts)
    cache.free([2])
    for l in range(L):
        for b, c in enumerate(counts):
            if c:
                rows[l][b] = [[x[0:2 * c:2] for x in unit] for unit in rows[l][b]]
                rows[l][b] = [[torch.cat([x, torch.zeros_like(x[:c - len(x)])]) for x in unit] for unit in rows[l][b]]
    got_k, got_v = cache.read([len(rows[0][b][0][0]) if b != 2 else 1 for b in range(batch)])
    lens = [len(rows[0][b][0][0]) if b != 2 else 1 for b in range(batch)]
    cu = R.cu_of(lens)
    for l in range(L):
        for b in range(batch):
            for h in range(HKV):
                for x, i in ((got_k, 0), (got_v, 1)):
                    want = rows[l][b][h][i].to(torch.bfloat16) if b != 2 else torch.zeros((1, d), dtype=torch.bfloat16, device="cuda")
                    assert torch.equal(x[l, cu[b]:cu[b + 1], h], want), (l, b, h, i)
    cache.free(range(batch))
    assert not cache.refs.any() and not cache.lens.any()
    with pytest.raises(M.MMShiftError):
        cache.poll()
    cache.poll()
    attention.poll()


def test_a_captured_step_of_all():
    """Positions, rotation, pages, rows and attention of a step in a graph, replayed as answers grow."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    d, batch = 64, 4
    rotary = Rotary(d)
    cache, plain = (PagedKVCache(HQ, HKV, d, torch.bfloat16, batch, 200, page_size=16, pages=80) for _ in range(2))
    k0, v0 = rnd(1, 60, HKV, d), rnd(1, 60, HKV, d)
    for c in (cache, plain):
        c.advance([60, 0, 0, 0])
        c.append(k0, v0, [60, 0, 0, 0])
        c.fork([0, 0, 0], [1, 2, 3])
    q, k, v = rnd(batch, HQ, d), rnd(batch, HKV, d), rnd(1, batch, HKV, d)
    pos = torch.full((batch,), 60, dtype=torch.int32, device="cuda")
    out = torch.empty((batch, HQ, d), dtype=torch.bfloat16, device="cuda")
    new = [1] * batch

    def step(c, result):
        a, b = rotary(q, k, pos)
        c.advance(new)
        c.append(b[None], v, new)
        c.attend(a, new, groups=[4], out=result)
        pos.add_(1)

    cache.attend(q, new, groups=[4])               # such a call has been made once before
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, out)
    want = torch.empty_like(out)
    for i in range(40):
        for x in (q, k, v):
            x.copy_(rnd(*x.shape))
        graph.replay()
        pos.sub_(1)
        step(plain, want)
        assert R.same(out, want), i
        assert torch.equal(cache.page_table, plain.page_table) and torch.equal(cache.refs, plain.refs)
    cache.poll()


def test_replays_report_after_larger_calls():
    """A graph's attention in groups goes on with the workspace it was captured with when a larger call
    has taken another: what a replay reports there is raised, once."""
    batch, new = 4, [1] * 4
    cache = PagedKVCache(HQ, HKV, 64, torch.bfloat16, batch, 200, page_size=16, pages=80)
    gen = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    cache.advance([60, 0, 0, 0])
    cache.append(rnd(1, 60, HKV, 64), rnd(1, 60, HKV, 64), [60, 0, 0, 0])
    cache.fork([0, 0, 0], [1, 2, 3])
    q, out = rnd(batch, HQ, 64), torch.empty((batch, HQ, 64), dtype=torch.bfloat16, device="cuda")
    graphs = []
    for more in (1, 20, 45):
        q_more = rnd(batch * more, HQ, 64)
        cache.attend(q_more, [more] * batch, groups=[4])   # a larger workspace each time
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            cache.attend(q, new, groups=[4], out=out)
    cache.poll()
    table = cache.page_table.clone()
    for g in graphs:
        g.replay()
        cache.poll()
        cache.page_table[0, 2, 1, 0] = -1              # a page that is not there
        g.replay()
        with pytest.raises(M.MMShiftError):
            cache.poll()
        cache.page_table.copy_(table)
        g.replay()
        cache.poll()


def test_what_was_reported_before_a_larger_call_is_raised():
    cache = PagedKVCache(HQ, HKV, 64, torch.bfloat16, 2, 200, page_size=16, pages=40)
    k = torch.zeros((1, 40, HKV, 64), dtype=torch.bfloat16, device="cuda")
    cache.advance([20, 20])
    cache.append(k, k, [20, 20])
    cache.page_table[0, 1, 0, 0] = -1
    for n in (1, 15):
        cache.attend(torch.zeros((2 * n, HQ, 64), dtype=torch.bfloat16, device="cuda"), [n] * 2, groups=[2])
    cache.page_table[0, 1, 0, 0] = cache.page_table[0, 1, 0, 1]
    cache.attend(torch.zeros((80, HQ, 64), dtype=torch.bfloat16, device="cuda"), [40] * 2, groups=[2])
    with pytest.raises(M.MMShiftError):
        cache.poll()
    cache.poll()
