"""Attention over whole prompts against its formula in float64, element by element within
the bounds of tests/cache_ref.py (whose derivation holds for any rows of keys)."""
import math

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300.prompt import PromptAttention
from tests import cache_ref as R

pytestmark = pytest.mark.gpu


def reference(q, k, v, cu, causal, scale=0.0):
    """out, lse and their tolerances, as cache_ref.reference's for each row."""
    T, hq, d = q.shape
    hkv = k.shape[1]
    r = hq // hkv
    bf = q.dtype == torch.bfloat16
    scale = scale or 1.0 / math.sqrt(d)
    out, tol = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    ltol = torch.zeros_like(lse)
    for a, b in zip(cu, cu[1:]):
        n = b - a
        if n == 0:
            continue
        seen = torch.ones((n, n), dtype=torch.bool, device="cuda")
        if causal:
            seen = seen.tril()
        count = seen.sum(-1).double()[:, None]
        for h in range(hkv):
            kk, vv = k[a:b, h].double(), v[a:b, h].double()
            for j in range(h * r, (h + 1) * r):
                x = q[a:b, j].double()
                z = torch.where(seen, x @ kk.T * scale, -math.inf)
                zerr = ((d + 4) * R.U32 * (x.abs() @ kk.abs().T) * scale).masked_fill(~seen, 0).nan_to_num(0, 0, 0).amax(-1)
                top = torch.logsumexp(z, -1)
                p = torch.softmax(z, -1)
                lse[a:b, j] = torch.where(top == math.inf, math.nan, top)
                worst = z.masked_fill(~seen, 0).abs().nan_to_num(0, 0, 0).amax(-1)
                ltol[a:b, j] = zerr + (8 + count[:, 0]) * R.U32 + 2 * R.U32 * (worst + 1)
                # keys that a row does not see have no part in it, whatever they hold
                w = torch.where(p == 0, 0, 1).bool() | seen
                o, mean = torch.zeros_like(x), torch.zeros_like(x)
                odd = ~torch.isfinite(vv).all(-1)
                clean = torch.where(torch.isfinite(vv), vv, 0.0)
                o, mean = p @ clean, p @ clean.abs()
                for t in odd.nonzero()[:, 0].tolist():
                    bad = torch.where(torch.isfinite(vv[t]), 0.0, vv[t])
                    o = torch.where((seen[:, t] & w[:, t])[:, None] & ~torch.isfinite(vv[t])[None], o + p[:, t:t + 1] * bad, o)
                rel = 4 * zerr + (16 + 2 * count[:, 0]) * R.U32 + (R.UBF + R.U32 if bf else 0)
                out[a:b, j] = o
                tol[a:b, j] = rel[:, None] * mean + (R.UBF if bf else R.U32) * o.abs() + 1e-37
    return out, lse, tol * 1.01, ltol * 1.01


def rows(cu, hq, hkv, d, dtype, seed=0, spread=1.0, strided=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T = cu[-1]
    if strided:
        x = torch.randn((T, (hq + 2 * hkv) * d + 8), generator=gen, device="cuda").to(R.DT[dtype])
        q, k, v = (y.unflatten(-1, (-1, d)) for y in x[:, :-8].split([hq * d, hkv * d, hkv * d], -1))
        return q, k, v
    q, k, v = (torch.randn((T, h, d), generator=gen, device="cuda").to(R.DT[dtype]) for h in (hq, hkv, hkv))
    return q * spread, k, v


def run(q, k, v, cu, causal=True, scale=0.0, status=M._lib.MMSHIFT_OK):
    at = PromptAttention(q.shape[1], k.shape[1], q.shape[2], q.dtype, cu)
    n = at._ws_bytes
    at._workspace = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")   # only the status word is zero
    at._workspace[:256].zero_()
    out = torch.full(q.shape, math.nan, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], math.nan, device="cuda")
    at(q, k, v, causal, scale, out=out, lse=lse)
    assert M.mmshift_poll_status(at._workspace) == status
    assert (at._workspace[n:] == 0xA5).all()
    return out, lse


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (4, 4, 128), (8, 1, 64), (6, 2, 64), (5, 1, 128), (40, 1, 64)])
@pytest.mark.parametrize("lens", [[1], [2, 1, 0, 3], [127, 128, 129], [300, 0, 17, 64, 255]])
def test_lengths(causal, hq, hkv, d, lens):
    cu = R.cu_of(lens)
    x = rows(cu, hq, hkv, d, "bf16", seed=sum(lens))
    R.check_attention(run(*x, cu, causal), reference(*x, cu, causal), (causal, hq, hkv, d, lens))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,d,lens", [(4, 2, 64, [1, 0, 33, 130]), (3, 3, 128, [257]), (7, 1, 64, [65, 64, 63, 1])])
def test_float32(causal, hq, hkv, d, lens):
    cu = R.cu_of(lens)
    for strided in (False, True):
        x = rows(cu, hq, hkv, d, "f32", seed=3, strided=strided)
        R.check_attention(run(*x, cu, causal), reference(*x, cu, causal), (causal, hq, hkv, d, lens))


def test_longer_prompts():
    """Runs of many tiles, and units shared by several CTAs."""
    for hq, hkv, d, lens, causal in ((2, 1, 128, [3001], True), (7, 1, 128, [1500, 70, 900], True), (2, 2, 64, [2500], False),
                                     (16, 16, 64, [600, 1], True)):
        cu = R.cu_of(lens)
        x = rows(cu, hq, hkv, d, "bf16", seed=9, spread=3.0)
        R.check_attention(run(*x, cu, causal), reference(*x, cu, causal), (hq, hkv, d, lens))


def test_many_prompts_of_few_tokens():
    lens = [(i * 7) % 23 for i in range(64)]
    cu = R.cu_of(lens)
    for hq, hkv in ((28, 4), (8, 8)):
        x = rows(cu, hq, hkv, 128, "bf16", seed=2)
        R.check_attention(run(*x, cu), reference(*x, cu, True), (hq, hkv))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_scales_and_results_without_lse(dtype):
    cu = R.cu_of([150, 33])
    x = rows(cu, 6, 2, 64, dtype, seed=4, strided=True)
    for scale in (0.05, 3.0):
        R.check_attention(run(*x, cu, True, scale), reference(*x, cu, True, scale), scale)
    at = PromptAttention(6, 2, 64, x[0].dtype, cu)
    assert R.same(at(*x), run(*x, cu)[0])
    # a query and a result that start anywhere
    T = cu[-1]
    buf = torch.empty(T * 6 * 64 + 1, dtype=x[0].dtype, device="cuda")
    out, q = buf[1:].view(T, 6, 64), torch.empty_like(buf)[1:].view(T, 6, 64).copy_(x[0])
    at(q, x[1], x[2], out=out)
    assert R.same(out.clone(), at(*x))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
def test_values_that_are_not_finite(dtype, causal):
    """NaN and infinities reach the rows that attend to them and no others, not those of the next prompt."""
    cu = R.cu_of([140, 100, 300])
    q, k, v = rows(cu, 4, 2, 64, dtype, seed=6)
    v[139, 0, 5] = math.nan                        # the last of a prompt
    v[140 + 20, 1, 60] = math.inf
    v[240 + 131, 0, 0] = -math.inf
    v[240 + 131, 0, 63] = math.nan
    v[240 + 200, 1, 7] = math.inf
    got, want = run(q, k, v, cu, causal), reference(q, k, v, cu, causal)
    R.check_attention(got, want, "values")
    k[100, 1, 3] = math.nan
    k[300, 0, 3] = math.inf
    q[50, 0, 1] = math.inf
    got = run(q, k, v, cu, causal)
    want = reference(q, k, v, cu, causal)
    # rows with a NaN or +inf among their logits are NaN, whatever their values are
    bad = torch.isnan(want[1])
    assert torch.equal(torch.isnan(got[1]), bad) and torch.isnan(got[0][bad]).all()
    for i in (0, 2):
        want[i][bad] = 0
    R.check_attention((got[0].masked_fill(bad[..., None], 0), got[1].masked_fill(bad, 0)),
                      (want[0], want[1].masked_fill(bad, 0), want[2], want[3]), "keys")


def test_logits_of_minus_infinity():
    cu = R.cu_of([200])
    q, k, v = rows(cu, 2, 1, 64, "bf16", seed=8)
    q[:, :, 0] = q[:, :, 0].abs() + 1
    k[:150, :, 0] = -math.inf
    k[150:, :, 0] = 1
    got, want = run(q, k, v, cu), reference(q, k, v, cu, True)
    want[0][:150], want[2][:150] = 0, 0            # rows that see such keys alone
    R.check_attention(got, want, "minus infinity")


def test_a_prompt_is_a_cache_of_its_own_rows():
    """The same rows through the paged cache's attention."""
    n = 333
    q, k, v = rows([0, n], 6, 2, 128, "bf16", seed=11)
    cache = R.Cache([[n, n]], 128, "bf16", 64)
    for h in range(2):
        cache.put(0, 0, h, torch.arange(n), k[:, h], v[:, h])
    a, b = run(q, k, v, [0, n]), R.attend(cache, q, [n])
    want = reference(q, k, v, [0, n], True)
    R.check_attention(a, want)
    R.check_attention(b, want)


def test_captured_and_on_another_stream():
    cu = R.cu_of([70, 200])
    x = rows(cu, 8, 2, 64, "bf16", seed=12)
    at = PromptAttention(8, 2, 64, torch.bfloat16, cu)
    want = at(*x).clone()
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        at(*x, out=out)
    side.synchronize()
    assert R.same(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        at(*x, out=out)
    out.zero_()
    graph.replay()
    assert R.same(out, want)
    for t in x:
        t.mul_(-0.5)
    graph.replay()
    assert R.same(out, at(*x))
    at.poll()


def test_repeated_calls_are_equal():
    cu = R.cu_of([900, 1300])
    x = rows(cu, 28, 4, 128, "bf16", seed=13)
    a = run(*x, cu)
    for _ in range(3):
        b = run(*x, cu)
        assert R.same(a[0], b[0]) and R.same(a[1], b[1])


def test_more_heads_than_a_block_has_rows():
    """A token's query heads in several blocks."""
    for hq, d, lens in ((130, 64, [3, 40]), (200, 128, [17])):
        cu = R.cu_of(lens)
        x = rows(cu, hq, 1, d, "bf16", seed=14)
        R.check_attention(run(*x, cu), reference(*x, cu, True), (hq, d))


def test_rows_past_four_gigabytes():
    lens, hq, hkv, d, width = [33000, 130], 2, 1, 64, 70000
    cu = R.cu_of(lens)
    buf = torch.empty((cu[-1], width), dtype=torch.bfloat16, device="cuda")
    assert buf[-130:].data_ptr() - buf.data_ptr() > 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(15)
    at = width - (hq + 2 * hkv) * d
    buf[:, at:] = torch.randn((cu[-1], width - at), generator=gen, device="cuda").bfloat16()
    q, k, v = (x.unflatten(-1, (-1, d)) for x in buf[:, at:].split([hq * d, hkv * d, hkv * d], -1))
    out, lse = run(q, k, v, cu)
    want = reference(q[-130:], k[-130:], v[-130:], [0, 130], True)
    R.check_attention((out[-130:], lse[-130:]), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_many_units_a_worker(d, causal):
    """Units of one and of two blocks, of one key tile and of several, one after the other."""
    lens = [17, 300, 1, 500, 64, 333, 129, 5, 260, 2, 350, 90, 0, 18]
    cu = R.cu_of(lens)
    x = rows(cu, 112, 16, d, "bf16", seed=16, spread=2.0)
    R.check_attention(run(*x, cu, causal), reference(*x, cu, causal), (d, causal))
