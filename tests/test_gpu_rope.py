"""Rotary positions against the formula in float64."""
import math

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300.prompt import Rotary
from tests import cache_ref as R

pytestmark = pytest.mark.gpu

# The angle: 2^-32 turns cut off, and as a float32 of at most one half turn 2^-26 turns; its sine
# and cosine 2 units in the last place, and one more for the amplitude's product.
ANGLE = 2 * math.pi * (2.0 ** -26 + 2.0 ** -31) + 6 * R.U32


def reference(x, positions, freq, layout, sections, amplitude, inverse=False):
    """x [..., T, H, d], positions [axes, T]: the rotated rows and how far they may be off."""
    n = len(freq)
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections)).cuda()
    w = positions[axis].T.double() * torch.tensor(freq, dtype=torch.float64, device="cuda")
    c, s = (amplitude * f(w)[:, None] for f in (torch.cos, torch.sin))
    if inverse:
        s = -s
    y, tol = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    i = torch.arange(n, device="cuda")
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    xa, xb = x.double()[..., a], x.double()[..., b]
    y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
    u = R.UBF if x.dtype == torch.bfloat16 else R.U32
    for at in (a, b):
        tol[..., at] = amplitude * (xa.abs() + xb.abs()) * (ANGLE + 3 * R.U32) + u * y[..., at].abs() + 1e-37
    return y, tol * 1.01


def check(got, x, *a, **kw):
    want, tol = reference(x, *a, **kw)
    over = (got.double() - want).abs() > tol
    assert not over.any(), (int(over.sum()), over.nonzero()[:4].tolist(), float((got.double() - want).abs().max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot,sections", [(128, 128, None), (64, 64, None), (128, 64, (5, 11, 16)), (64, 48, (0, 24)),
                                            (128, 96, None), (64, 24, (12, 0, 0)), (128, 2, None), (64, 32, None)])
def test_rows(dtype, layout, d, rot, sections):
    gen = torch.Generator(device="cuda").manual_seed(d + rot)
    for hq, hkv, T, L in ((28, 4, 5, 1), (6, 6, 37, 2), (1, 1, 1, 1), (40, 8, 300, 1)):
        x, y = (torch.randn((L, T, h, d), generator=gen, device="cuda").to(R.DT[dtype]) for h in (hq, hkv))
        axes = 1 if sections is None else len(sections)
        pos = torch.randint(-3000, 3000000, (axes, T), generator=gen, device="cuda", dtype=torch.int32)
        rotary = Rotary(d, rot, 1e6, layout, sections, amplitude=1.25)
        args = (pos, rotary.inv_freq, layout, sections or (rot // 2,), 1.25)
        q, k = rotary(x, y, pos if axes > 1 else pos[0])
        check(q, x, *args)
        check(k, y, *args)
        q2, k2 = rotary(x.clone(), y.clone(), pos if axes > 1 else pos[0], in_place=True)
        assert R.same(q, q2) and R.same(k, k2)
        back, _ = rotary(x, y, pos if axes > 1 else pos[0], inverse=True)
        check(back, x, *args, inverse=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_strides_and_alignment(dtype, layout, shift):
    """Q and K inside a projection's rows, which start anywhere: only their elements change."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    T, hq, hkv, d, L = 23, 12, 4, 64, 2
    for width in ((hq + 2 * hkv) * d, (hq + 2 * hkv) * d + 3):
        buf = torch.randn((L * T * width + 16,), generator=gen, device="cuda").to(R.DT[dtype])
        rows = buf[shift:shift + L * T * width].view(L, T, width)
        before = rows.clone()
        q, k = rows[..., :hq * d].unflatten(-1, (hq, d)), rows[..., hq * d:(hq + hkv) * d].unflatten(-1, (hkv, d))
        pos = torch.randint(0, 40000, (T,), generator=gen, device="cuda", dtype=torch.int32)
        rotary = Rotary(d, layout=layout)
        args = (pos[None], rotary.inv_freq, layout, (d // 2,), 1.0)
        q1, k1 = rotary(q, k, pos)
        assert R.same(rows.contiguous(), before)
        check(q1, q, *args)
        check(k1, k, *args)
        rotary(q, k, pos, in_place=True)
        assert R.same(q.contiguous(), q1) and R.same(k.contiguous(), k1)
        assert R.same(rows[..., (hq + hkv) * d:].contiguous(), before[..., (hq + hkv) * d:].contiguous())


def test_one_side_and_heads_of_any_number():
    gen = torch.Generator(device="cuda").manual_seed(5)
    pos = torch.arange(9, dtype=torch.int32, device="cuda")
    rotary = Rotary(128)
    args = (pos[None], rotary.inv_freq, "half", (64,), 1.0)
    for hq, hkv in ((5, None), (None, 3), (5, 3)):
        q, k = (None if h is None else torch.randn((9, h, 128), generator=gen, device="cuda").bfloat16() for h in (hq, hkv))
        for got, x in zip(rotary(q, k, pos), (q, k)):
            assert (got is None) == (x is None)
            if x is not None:
                check(got, x, *args)


def test_far_positions_turn_exactly():
    """Frequencies of whole fractions of a turn come round, at the farthest positions too."""
    n = 32
    freq = [2 * math.pi * (2 * j + 1) / 64 for j in range(n)]          # 64 positions: whole turns
    x = torch.randn((4, 1, 2 * n), device="cuda")
    pos = torch.tensor([3, 3 + 64 * 1000003, 3 - 2 ** 31 + 64, 2 ** 31 - 64 + 3], dtype=torch.int32, device="cuda")
    x[1:] = x[0]
    got, _ = Rotary(2 * n, inv_freq=freq)(x, None, pos)
    # the fraction of a turn is a double: 2^31 positions add up 2^31 times 2^-53 turns of it
    assert (got - got[0]).abs().max() < 2 * float(x.abs().max()) * (ANGLE + 2 * math.pi * 2.0 ** -21)


def test_scalings_against_their_formulas():
    for scaling in ("none", "linear", "base", "parts"):
        r = Rotary(64, 0, 1e4, scaling=scaling, factor=1.0 if scaling == "none" else 8.0, original_length=4096)
        f = [1e4 ** (-j / 32) for j in range(32)]
        if scaling == "linear":
            f = [x / 8 for x in f]
        if scaling == "base":
            f = [(1e4 * 8 ** (64 / 62)) ** (-j / 32) for j in range(32)]
        if scaling == "parts":
            ramp = [min(max((4096 * x / (2 * math.pi) - 1) / 31, 0), 1) for x in f]
            f = [x * r_ + x / 8 * (1 - r_) for x, r_ in zip(f, ramp)]
            assert abs(r.amplitude - (0.1 * math.log(8) + 1)) < 1e-6
        else:
            assert r.amplitude == 1.0
        assert max(abs(a - b) / b for a, b in zip(r.inv_freq, f)) < 1e-13


def test_the_gradient_is_the_other_turn():
    """d/dx of <g, rotate(x)> against the other way's rotation of g, and against differences."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, g = (torch.randn((7, 3, 64), generator=gen, device="cuda") for _ in range(2))
    pos = torch.randint(0, 100000, (7,), generator=gen, device="cuda", dtype=torch.int32)
    r = Rotary(64, 48, amplitude=1.5)
    back, _ = r(g, None, pos, inverse=True)
    base = (r(x, None, pos)[0].double() * g).sum()
    # linear in x: a difference is exact but for rounding (3 U32 a term, two rotations)
    for step in range(4):
        dx = torch.randn(x.shape, generator=gen, device="cuda")
        diff = (r(x + dx, None, pos)[0].double() * g).sum() - base
        moved = ((x + dx).double() - x.double())
        tol = 2 * 1.5 * ((x.abs() + (x + dx).abs() + dx.abs()).double().sum() * g.abs().max()) * (ANGLE + 8 * R.U32)
        assert abs(float(diff - (back.double() * moved).sum())) < float(tol)


def test_captured():
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    x = torch.randn((3, 2, 64), device="cuda")
    y = x.clone()
    r = Rotary(64)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got, _ = r(x, None, pos)
    for p in ([0, 1, 2], [7, 100000, 5]):
        pos.copy_(torch.tensor(p, dtype=torch.int32))
        graph.replay()
        check(got, y, pos[None], r.inv_freq, "half", (32,), 1.0)


def test_nothing_to_rotate():
    r = Rotary(64)
    q, k = r(torch.empty((0, 4, 64), device="cuda"), torch.empty((0, 2, 64), device="cuda"),
             torch.empty(0, dtype=torch.int32, device="cuda"))
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_layers_side_by_side_in_a_token(dtype, pad):
    """[T, L, heads, d] buffers as [L, T, heads, d]: only their rows change in place."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    hq, hkv, d = 12, 4, 64
    for T, L in ((37, 3), (1, 2), (2, 5), (300, 2)):
        rows = torch.randn((T, L, (hq + hkv) * d + pad), generator=gen, device="cuda").to(R.DT[dtype])
        before = rows.clone()
        q, k = (x.unflatten(-1, (h, d)).transpose(0, 1) for x, h in ((rows[..., :hq * d], hq), (rows[..., hq * d:(hq + hkv) * d], hkv)))
        pos = torch.randint(0, 40000, (T,), generator=gen, device="cuda", dtype=torch.int32)
        rotary = Rotary(d)
        args = (pos[None], rotary.inv_freq, "half", (d // 2,), 1.0)
        q1, k1 = rotary(q, k, pos)
        assert R.same(rows, before)
        check(q1, q, *args)
        check(k1, k, *args)
        rotary(q, k, pos, in_place=True)
        assert R.same(q.contiguous(), q1) and R.same(k.contiguous(), k1)
        assert R.same(rows[..., (hq + hkv) * d:].contiguous(), before[..., (hq + hkv) * d:].contiguous())


def test_rows_that_require_a_gradient_where_none_is_recorded():
    x = torch.randn((5, 2, 64), device="cuda", requires_grad=True)
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    r = Rotary(64)
    with torch.no_grad():
        a, _ = r(x, None, pos)
    b, _ = r(x.detach(), None, pos)
    assert R.same(a, b) and not a.requires_grad
    with pytest.raises(ValueError, match="gradient"):
        r(x, None, pos)
