"""Attention's weights at the ends of their types' range: one key far above the others, values
whose magnitudes differ by many powers of two from row to row."""
import math

import pytest
import torch

from tests import cache_ref as R

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")]


def _check(cache, q, new):
    """Within cache_ref's bounds and, for few rows over 8-bit pages, what float16 weights add:
    2^-32 of a row's largest product of weight and scale for every key (half of float16's last
    step, 2^-25, where that product is held at 2^7 or above), times the key's codes."""
    out, lse, tol, ltol = R.reference(cache, q, new)
    r = q.shape[1] // cache.H
    if cache.kind == "i8" and q.dtype == torch.bfloat16:
        cu = R.cu_of(new)
        for b, n in enumerate(new):
            for h in range(cache.H if n * r <= 32 else 0):
                m = int(cache.lens_host[0, b, h])
                for i in range(n):
                    pos = torch.arange(m - n + i + 1)
                    if not len(pos):
                        continue
                    k, v = cache.get(0, b, h, pos)
                    vs = cache.vs.view(-1)[cache.slots(0, b, h, pos)].double()
                    codes = cache.vp.view(-1, cache.d)[cache.slots(0, b, h, pos)].double().abs().sum(0)
                    p = torch.softmax(q[cu[b] + i, h * r:(h + 1) * r].double() @ k.T / math.sqrt(cache.d), -1)
                    tol[cu[b] + i, h * r:(h + 1) * r] += 2.0 ** -32 * (p * vs).amax(-1, keepdim=True) * codes
    R.check_attention(R.attend(cache, q, new), (out, lse, tol, ltol))


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,rows", [(1, 3000), (2, 1500), (9, 700), (40, 700)])
@pytest.mark.parametrize("gap", [9.0, 14.0, 17.0, 18.5])
def test_one_key_far_above_the_others(dtype, kind, d, n, rows, gap):
    """The first key's logit lies `gap` above all others', and its values are zero in half of the
    dimensions: what stands there is the sum of the others' small weights."""
    cache = R.Cache([[rows]], d, kind, 16)
    gen = torch.Generator(device="cuda").manual_seed(int(gap))
    k, v = (torch.randn((rows, d), generator=gen, device="cuda") for _ in range(2))
    k[:, 0], k[0, 0] = 0, gap / 8
    k[0, 1:] *= gap / 40                               # its largest stays the first
    v = 1 + 0.1 * v
    v[0, ::2] = 0
    cache.put(0, 0, 0, torch.arange(rows), k, v)
    q = torch.zeros((n, 3, d), device="cuda")
    q[..., 0] = 8 * math.sqrt(d)
    _check(cache, q.to(R.DT[dtype]), [n])


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 5, 40])
@pytest.mark.parametrize("outlier", [0, 12, 22, 30])
def test_values_of_many_magnitudes(dtype, kind, d, n, outlier):
    """Rows of V over several decades, and one with a single value 2^outlier above them."""
    cache = R.Cache([[300, 90], [513, 41]], d, kind, 16).fill_random(3)
    gen = torch.Generator(device="cuda").manual_seed(outlier)
    for b in range(2):
        for h in range(2):
            m = int(cache.lens_host[0, b, h])
            k, v = cache.get(0, b, h, torch.arange(m))
            v = v * torch.exp(3 * torch.randn((m, 1), generator=gen, device="cuda"))
            if outlier:
                v[m // 3] = 0
                v[m // 3, 7] = 2.0 ** outlier
            cache.put(0, b, h, torch.arange(m), k, v)
    _check(cache, torch.randn((2 * n, 6, d), generator=gen, device="cuda").to(R.DT[dtype]), [n, n])
