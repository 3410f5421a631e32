"""Attention calls in which a CTA has many units in turn (runs): chunks of at most 128 rows
of a KV head, whose blocks take the runs in turn, beside longer ones, and more runs than are
listed ahead. Against the formula in float64, with garbage behind every sequence's end."""
import math
import random

import pytest
import torch

from tests import cache_ref as R

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")]


def _reference(cache, q, new):
    """cache_ref.reference under the causal mask, a sequence at a time: the same values and bounds."""
    d, r, bf = cache.d, q.shape[1] // cache.H, q.dtype == torch.bfloat16
    scale, cu = 1.0 / math.sqrt(d), R.cu_of(new)
    out, tol = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    ltol = torch.zeros_like(lse)
    for b, n in enumerate(new):
        for h in range(cache.H):
            m = int(cache.lens_host[0, b, h])
            if not (n and m):
                continue
            k, v = cache.get(0, b, h, torch.arange(m))
            x = q[cu[b]:cu[b + 1], h * r:(h + 1) * r].double()                      # [n, r, d]
            end = (m - n + 1 + torch.arange(n, device="cuda")).clamp(min=0)
            seen = (torch.arange(m, device="cuda") < end[:, None])[:, None]         # [n, 1, m]
            z = x @ k.T * scale
            size = z.abs().masked_fill(~seen, 0).amax(-1)
            zerr = ((d + 4) * R.U32 * (x.abs() @ k.abs().T) * scale).masked_fill(~seen, 0).amax(-1)
            z = z.masked_fill(~seen, -math.inf)
            p = torch.softmax(z, -1).nan_to_num(0)                                  # rows without keys
            at = (slice(cu[b], cu[b + 1]), slice(h * r, (h + 1) * r))
            lse[at] = torch.logsumexp(z, -1)
            ltol[at] = zerr + ((8 + end) * R.U32)[:, None] + 2 * R.U32 * (size + 1)
            out[at] = p @ v
            rel = 4 * zerr + ((16 + 2 * end) * R.U32)[:, None] + (R.UBF + R.U32 if bf else 0)
            tol[at] = rel[..., None] * (p @ v.abs()) + (R.UBF if bf else R.U32) * out[at].abs() + 1e-37
    return out, lse, tol * 1.01, ltol * 1.01


def _run(lens, new, hq, d, dtype, kind, page, times=3):
    cache = R.Cache(lens, d, kind, page, seed=d).fill_random(7)
    gen = torch.Generator(device="cuda").manual_seed(8)
    q = torch.randn((sum(new), hq, d), generator=gen, device="cuda").to(R.DT[dtype])
    before, want = cache.clone_tensors(), _reference(cache, q, new)
    first = R.attend(cache, q, new)
    R.check_attention(first, want)
    for _ in range(times - 1):
        again = R.attend(cache, q, new)
        assert R.same(again[0], first[0]) and R.same(again[1], first[1])
    for a, b in zip(cache.tensors(), before):
        assert R.same(a, b)


def test_the_reference_is_the_slow_one():
    cache = R.Cache([[40, 7], [3, 90]], 64, "bf16", 16).fill_random()
    q = torch.randn((14, 6, 64), device="cuda").bfloat16()
    got, want = _reference(cache, q, [9, 5]), R.reference(cache, q, [9, 5])
    keys = torch.isfinite(want[1])                     # of rows without keys no bound is asked
    assert torch.equal(keys, torch.isfinite(got[1])) and not keys.all()
    for a, b in zip(got, want):
        assert torch.allclose(a[keys], b[keys], rtol=1e-9, atol=1e-30)


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,batch,hq,hkv", [(1000, 16, 28, 4), (700, 8, 28, 4), (600, 16, 32, 32)])
def test_fresh_prompts(kind, d, n, batch, hq, hkv):
    """Sequences that hold a prompt's own rows and no others: the first tiles of a head are masked
    from their first key on, its last rows fill half a tile."""
    _run([[n] * hkv] * batch, [n] * batch, hq, d, "bf16", kind, 64)


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [8, 10])
def test_drafts_over_heads_with_budgets(kind, d, n):
    rng = random.Random(n)
    lens = [[rng.randint(64, 2048) for _ in range(4)] for _ in range(64)] if n == 8 else [[1500] * 4, [60] * 4] * 32
    _run(lens, [n] * 64, 28, d, "bf16", kind, 32)


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("long", [1100, 2300])
def test_long_and_short_sequences_in_turn(kind, d, long):
    _run([[long] * 8, [64] * 8] * 32, [64] * 64, 8, d, "bf16", kind, 16)


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("d", [64, 128])
def test_short_chunks_beside_long_ones(kind, d):
    """Units of one block next to units of two."""
    new = [40, 300, 17, 1000, 128, 129] * 4
    lens = [[n + (37 * i + 211 * h) % 900 * (i % 3 > 0) for h in range(3)] for i, n in enumerate(new)]
    _run(lens, new, 6, d, "bf16", kind, 16)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_more_runs_than_are_listed(dtype, kind, d):
    """2,816 units of 45 rows (float32: 72, more than the few rows' kernels take) over at most 22
    keys: 18 runs a CTA, where 16 are listed ahead."""
    B, H, n = 64, 44, 5 if dtype == "bf16" else 8
    lens = [[(5 * b + 7 * h) % 23 for h in range(H)] for b in range(B)]
    _run(lens, [n] * B, H * 9, d, dtype, kind, 16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,lens,hq,hkv", [
    ([1000] * 16, [[1000] * 4] * 16, 28, 4),
    ([64] * 64, [[2300] * 8, [64] * 8] * 32, 8, 8),
    ([10] * 64, [[1500] * 4, [60] * 4] * 32, 28, 4)])
def test_not_finite_values_reach_only_their_own_readers(d, new, lens, hq, hkv):
    """Values of the last tokens that are not finite: the tokens before them do not attend to
    them, so not a bit of their results may differ."""
    cache = R.Cache(lens, d, "bf16", 64).fill_random(7)
    gen = torch.Generator(device="cuda").manual_seed(8)
    q = torch.randn((sum(new), hq, d), generator=gen, device="cuda").bfloat16()
    want = R.attend(cache, q, new)
    for b in range(len(new)):
        for h in range(hkv):
            last = cache.slots(0, b, h, [lens[b][h] - 1])
            cache.vp.view(-1, d)[last, (7 * b + h) % d] = math.nan if b % 2 else math.inf
    out, lse = R.attend(cache, q, new)
    cu = R.cu_of(new)
    last = torch.zeros(sum(new), dtype=torch.bool, device="cuda")
    last[torch.tensor(cu[1:], device="cuda") - 1] = True
    assert R.same(out[~last], want[0][~last]) and R.same(lse, want[1])
    for b in range(len(new)):
        for h in range(hkv):
            x = out[cu[b + 1] - 1, h * (hq // hkv):(h + 1) * (hq // hkv)]
            bad = ~torch.isfinite(x)
            assert bad[:, (7 * b + h) % d].all() and int(bad.sum()) == hq // hkv


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("r", [17, 32, 33, 71, 128, 300])
def test_many_query_heads_of_one_kv_head(dtype, kind, d, r):
    """One token's rows are more than a tile of the few rows' kernels, or than a block's."""
    _run([[700], [1], [0], [129]], [1, 1, 1, 2], r, d, dtype, kind, 32)
