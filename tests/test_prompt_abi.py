"""Refusals of rotary positions and of attention over prompts: before anything is enqueued, so
without a GPU. No pointer here is dereferenced but the frequencies', which lie on the host."""
import ctypes
import math

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300 import _lib as L
from paper_2607_22586_gb300.prompt import PromptAttention, Rotary

FAKE = 1 << 40
BAD, UNSUPPORTED, WORKSPACE = L.MMSHIFT_ERR_INVALID_ARG, L.MMSHIFT_ERR_UNSUPPORTED, L.MMSHIFT_ERR_WORKSPACE


def _shape(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, window=2, dtype=0, cu_seqlens=[0, 3, 3, 10], budgets=[4, 1, 2])
    base.update(kw)
    return M.make_shape(**base)


BAD_ROWS = [
    (dict(n_q_heads=7), BAD), (dict(n_kv_heads=0), BAD), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(cu_seqlens=[0, 3, 2, 10]), BAD), (dict(cu_seqlens=[1, 3, 3, 10]), BAD),
    (dict(cu_seqlens=[0, 1, 1, 2 ** 27 + 1]), UNSUPPORTED),            # rows of all heads past 2^30
]


def _prompt(s=None, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=None, ws=FAKE, n=1 << 40, qs=0, ks=0, causal=1, scale=0.0):
    return M.mmshift_prompt_attention(s or _shape(), q, qs, k, v, ks, causal, scale, out, lse, ws, n)


@pytest.mark.parametrize("bad,code", BAD_ROWS + [(dict(n_layers=2), UNSUPPORTED)])
def test_bad_shapes(bad, code):
    s = _shape(**bad)
    assert _prompt(s) == code
    with pytest.raises(M.MMShiftError) as e:
        M.mmshift_prompt_workspace_size(s)
    assert e.value.code == code


@pytest.mark.parametrize("bad,code", [
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(out=None), BAD), (dict(ws=None), WORKSPACE),
    (dict(q=FAKE + 1), BAD), (dict(k=FAKE + 8), BAD), (dict(v=FAKE + 2), BAD), (dict(out=FAKE + 1), BAD),
    (dict(lse=FAKE + 2), BAD), (dict(qs=8 * 128 - 8), BAD), (dict(ks=2 * 128 - 8), BAD), (dict(ks=2 * 128 + 4), BAD),
    (dict(ks=1 << 38), BAD), (dict(causal=2), BAD), (dict(scale=-1.0), BAD), (dict(scale=math.nan), BAD),
    (dict(scale=2.0 ** 128 / 1.2), BAD), (dict(ws=FAKE + 128), WORKSPACE), (dict(n=255), WORKSPACE),
    (dict(n=M.mmshift_prompt_workspace_size(_shape()) - 1), WORKSPACE),
])
def test_bad_prompt_arguments(bad, code):
    assert _prompt(**bad) == code


def test_prompts_without_rows_are_no_error():
    s = _shape(cu_seqlens=[0, 0, 0, 0])
    n = M.mmshift_prompt_workspace_size(s)
    assert _prompt(s, n=n) == L.MMSHIFT_OK
    assert _prompt(s, q=None, k=None, v=None, out=None, n=n) == L.MMSHIFT_OK


def _rotary(n=64, positions=FAKE, **kw):
    freq = (ctypes.c_double * n)(*kw.pop("freq", [1.0 / (j + 1) for j in range(n)]))
    sections = (ctypes.c_int32 * 3)(*kw.pop("sections", (0, 0, 0)))
    r = L.Rotary(inv_freq=freq, positions=positions, sections=sections, **kw)
    r._freq = freq
    return r


def _rope(r, s=None, q=FAKE, k=FAKE + (1 << 36), oq=FAKE + (2 << 36), ok=FAKE + (3 << 36), qs=0, ql=0, ks=0, kl=0):
    return M.mmshift_rope(s or _shape(), r, q, qs, ql, k, ks, kl, oq, ok)


@pytest.mark.parametrize("bad,code", BAD_ROWS)
def test_bad_rope_shapes(bad, code):
    assert _rope(_rotary(), _shape(**bad)) == code


@pytest.mark.parametrize("bad", [
    dict(layout=2), dict(layout=-1), dict(rot_dims=1), dict(rot_dims=3), dict(rot_dims=130), dict(rot_dims=-2),
    dict(inverse=2), dict(n_axes=4), dict(n_axes=-1), dict(n_axes=2, sections=(32, 31, 0)),
    dict(n_axes=2, sections=(65, -1, 0)), dict(n_axes=3, sections=(2 ** 31 - 1, 2 ** 31 - 1, 66)),
    dict(amplitude=-1.0), dict(amplitude=math.nan), dict(amplitude=math.inf), dict(positions=None), dict(positions=FAKE + 2),
    dict(freq=[math.nan] * 64), dict(freq=[1.0] * 63 + [math.inf]),
])
def test_bad_rotations(bad):
    assert _rope(_rotary(**bad)) == BAD


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(oq=None), dict(k=None), dict(ok=None), dict(q=FAKE + 1), dict(ok=FAKE + (3 << 36) + 1),
    dict(qs=8 * 128 - 1), dict(ks=2 * 128 - 1), dict(q=None, oq=None, k=None, ok=None),
    dict(oq=FAKE + 2), dict(oq=FAKE - 10 * 8 * 128 * 2 + 2), dict(oq=FAKE + 10 * 8 * 128 * 2 - 2),   # overlaps what is read
    dict(s=_shape(n_layers=2), ql=10 * 8 * 128 - 1), dict(s=_shape(n_layers=2), kl=-1),
])
def test_bad_rope_arguments(bad):
    assert _rope(_rotary(), **bad) == BAD


def test_nothing_to_rotate_is_no_error():
    s = _shape(cu_seqlens=[0, 0, 0, 0])
    assert _rope(_rotary(positions=None), s, q=None, k=None, oq=None, ok=None) == L.MMSHIFT_OK
    assert M.mmshift_rope(s, None_rotary(), None, 0, 0, None, 0, 0, None, None) == BAD


def None_rotary():
    return L.Rotary()                              # no frequencies


@pytest.mark.parametrize("a", [
    dict(rot_dims=0), dict(rot_dims=3), dict(rot_dims=130), dict(theta=0.0), dict(theta=-1.0), dict(theta=math.inf),
    dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=math.nan), dict(scaling="base", rot_dims=2, factor=2.0),
    dict(scaling="parts", factor=2.0), dict(scaling="parts", factor=2.0, original_length=-1.0),
    dict(scaling="parts", factor=2.0, original_length=100.0, low_turns=3.0, high_turns=3.0),
])
def test_bad_frequencies(a):
    base = dict(rot_dims=64, theta=1e4)
    base.update(a)
    with pytest.raises(M.MMShiftError) as e:
        M.rope_frequencies(**base)
    assert e.value.code == BAD


def test_frequencies():
    f, a = M.rope_frequencies(64, 1e4)
    assert a == 1.0 and max(abs(x - 1e4 ** (-j / 32)) / x for j, x in enumerate(f)) < 1e-14
    f, a = M.rope_frequencies(64, 1e4, "parts", 4.0, 2048, 1.0, 4.0)
    for j, x in enumerate(f):
        y = 1e4 ** (-j / 32)
        keep = min(max((2048 * y / (2 * math.pi) - 1) / 3, 0), 1)
        assert abs(x - (y * keep + y / 4 * (1 - keep))) < 1e-14 * y
    assert abs(a - (0.1 * math.log(4) + 1)) < 1e-6


def test_classes_refuse():
    with pytest.raises(ValueError):
        Rotary(64, layout="both")(torch.zeros(1, 1, 64), None, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        Rotary(64, rot_dims=32, inv_freq=[1.0])
    with pytest.raises(ValueError):
        Rotary(64, scaling="other")
    r = Rotary(64)
    x, p = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32)
    for bad in (lambda: r(None, None, p), lambda: r(x, None, p), lambda: r(x[0], None, p)):   # no rows of a GPU
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):
        M.make_rotary([1.0], p.long())
    with pytest.raises(ValueError):
        M.make_rotary([1.0], p, sections=[1, 0])
    with pytest.raises(ValueError):
        M.make_rotary([1.0] * 4, p.view(3, 1), sections=[2, 2])
    with pytest.raises(ValueError):
        PromptAttention(4, 2, 64, torch.float16, [0, 3], device="cpu")
    with pytest.raises(M.MMShiftError):
        PromptAttention(4, 3, 64, torch.bfloat16, [0, 3], device="cpu")
    at = PromptAttention(4, 2, 64, torch.bfloat16, [0, 3], device="cpu")
    rows = lambda h, dt=torch.bfloat16: torch.zeros(3, h, 64, dtype=dt)  # noqa: E731
    for q, k, v in ((rows(4), rows(4), rows(2)), (rows(4)[:2], rows(2), rows(2)), (rows(4, torch.float32), rows(2), rows(2)),
                    (rows(4), rows(2), rows(4)[:, ::2]), (rows(4), rows(4)[:, :2], rows(2))):
        with pytest.raises(ValueError):
            at(q, k, v)


def test_layers_that_overlap_are_refused():
    """A layer stride of 0, one tensor for all layers, is no dense one. (Rotary._rotate: behind
    the check for rows of a GPU.)"""
    r, p = Rotary(64), torch.zeros(3, dtype=torch.int32)
    x = torch.zeros(5, 3, 2, 64)
    for t in (x[0].expand(5, 3, 2, 64), x[:, :1].expand(5, 3, 2, 64), torch.zeros(2000).as_strided((5, 3, 2, 64), (380, 128, 64, 1))):
        for q, k in ((t, None), (x, t)):
            with pytest.raises(ValueError):
                r._rotate(q, k, 2, 2, 5, 3, p, False, False)


def test_layers_side_by_side():
    """Layers inside a token's row do not overlap; one element less between them or between tokens, and they do.
    (Rotary._rotate: behind the check for rows of a GPU.)"""
    from paper_2607_22586_gb300.prompt import _layer_stride

    assert _layer_stride(torch.zeros(3, 5, 2, 64).transpose(0, 1), 5) == 128
    assert _layer_stride(torch.zeros(5000).as_strided((5, 3, 2, 64), (130, 700, 64, 1)), 5) == 130
    dense = 8 * 128
    for layer, row in ((dense - 1, 3 * dense), (dense, 3 * dense - 1), (dense + 1, 3 * dense), (1 << 62, 1 << 62)):
        if layer < 1 << 62:
            with pytest.raises(ValueError):
                _layer_stride(torch.zeros(40000).as_strided((3, 10, 8, 128), (layer, row, 128, 1)), 3)
        assert _rope(_rotary(), _shape(n_layers=3), qs=row, ql=layer) == BAD


def test_no_gradient_is_lost_without_a_word():
    """Rows that require a gradient are refused where gradients are recorded, before anything else."""
    r, at = Rotary(64), PromptAttention(4, 2, 64, torch.bfloat16, [0, 3], device="cpu")
    p = torch.zeros(3, dtype=torch.int32)
    rows = lambda h, grad: torch.zeros(3, h, 64, dtype=torch.bfloat16, requires_grad=grad)  # noqa: E731
    for i in range(3):
        q, k, v = (rows(h, j == i) for j, h in enumerate((4, 2, 2)))
        with pytest.raises(ValueError, match="gradient"):
            at(q, k, v)
        if i < 2:
            with pytest.raises(ValueError, match="gradient"):
                r(q, k, p)
            with pytest.raises(ValueError, match="gradient"):
                r(q if i == 0 else None, k if i == 1 else None, p)
            with torch.no_grad(), pytest.raises(ValueError, match="one GPU"):   # the next check
                r(q, k, p)
            with pytest.raises(ValueError, match="one GPU"):
                r(q.detach(), k.detach(), p)


def test_an_output_where_the_other_side_lies():
    """A dense output over the other side's rows, or over its output, would be read or written in any order."""
    T, hq, hkv, esz = 10, 8 * 128, 2 * 128, 2
    q, k = FAKE, FAKE + (1 << 36)
    ends = T * hq * esz, T * hkv * esz
    for oq, ok in ((k, None), (k + ends[1] - 2, None), (k - ends[0] + 2, None), (None, q), (None, q + ends[0] - 2),
                   (None, q - ends[1] + 2), (FAKE + (2 << 36), FAKE + (2 << 36)),
                   (FAKE + (2 << 36), FAKE + (2 << 36) + ends[0] - 2), (FAKE + (2 << 36), FAKE + (2 << 36) - ends[1] + 2),
                   (k, q)):
        assert _rope(_rotary(), oq=FAKE + (4 << 36) if oq is None else oq, ok=FAKE + (5 << 36) if ok is None else ok) == BAD
    assert _rope(_rotary(), oq=k, ok=k) == BAD            # K in place, Q's output over it
    assert _rope(_rotary(), oq=q, ok=q) == BAD            # Q in place, K's output over it
    # K's second layer, and not what lies between its layers
    s = _shape(n_layers=2)
    assert _rope(_rotary(), s, kl=1 << 30, oq=k + (2 << 30) - 2) == BAD
    assert _rope(_rotary(), s, kl=1 << 30, oq=k + (2 << 30) - 2 * ends[0] + 2) == BAD


def test_outputs_next_to_the_other_side_are_no_error():
    """What ends where the other begins passes the checks (there are no tokens to rotate, or there is no GPU)."""
    T, hq, hkv, esz = 10, 8 * 128, 2 * 128, 2
    q, k = FAKE, FAKE + (1 << 36)
    if torch.cuda.is_available():
        pytest.skip("the addresses are none")
    for oq, ok in ((k + T * hkv * esz, FAKE + (3 << 36)), (k - T * hq * esz, FAKE + (3 << 36)),
                   (FAKE + (2 << 36), FAKE + (2 << 36) + T * hq * esz), (q, k)):
        assert _rope(_rotary(), oq=oq, ok=ok) not in (BAD, UNSUPPORTED)
    assert _rope(_rotary(), _shape(cu_seqlens=[0, 0, 0, 0]), oq=k, ok=q) == L.MMSHIFT_OK
    assert _rope(_rotary(), _shape(n_layers=2), kl=1 << 30, oq=k + (1 << 30)) not in (BAD, UNSUPPORTED)


def test_rows_of_both_sides_in_place():
    """One token's rows turned as Q's and as K's would turn twice, or be written over."""
    for k in (FAKE, FAKE + 8 * 128 * 2 - 2, FAKE - 2 * 128 * 2 + 2):
        assert _rope(_rotary(), k=k, oq=FAKE, ok=k, qs=4096, ks=4096) == BAD
    if not torch.cuda.is_available():                  # the addresses are none: side by side they pass the checks
        for k in (FAKE + 8 * 128 * 2, FAKE - 2 * 128 * 2):
            assert _rope(_rotary(), k=k, oq=FAKE, ok=k, qs=4096, ks=4096) != BAD


def test_no_amplitude_stands_for_another():
    """The C struct's 0 is 1, a caller's 0 would be rows of zeros."""
    p = torch.zeros(3, dtype=torch.int32)
    for a in (0.0, -1.0, math.nan):
        with pytest.raises(ValueError):
            M.make_rotary([1.0], p, amplitude=a)
    assert M.make_rotary([1.0], p, amplitude=0.5).amplitude == 0.5 and M.make_rotary([1.0], p).amplitude == 1.0


def test_outputs_between_rows_are_no_error():
    """A dense output in the gap between two rows, or two layers, of what is read lies on none of them."""
    if torch.cuda.is_available():
        pytest.skip("the addresses are none")
    s = _shape(cu_seqlens=[0, 1, 1, 2])
    q, k, gap = FAKE, FAKE + (1 << 36), 1 << 20            # elements between tokens
    dense = 2 * 8 * 128 * 2
    for oq in (k + 2 * 128 * 2, k + gap * 2 - dense, q + 8 * 128 * 2, q + gap * 2 - dense):
        assert _rope(_rotary(), s, qs=gap, ks=gap, oq=oq) not in (BAD, UNSUPPORTED)
    for oq in (k + 2 * 128 * 2 - 2, k + gap * 2 - dense + 2, q + 8 * 128 * 2 - 2, q + gap * 2 - dense + 2, k + gap * 2):
        assert _rope(_rotary(), s, qs=gap, ks=gap, oq=oq) == BAD
    assert _rope(_rotary(), s, ks=gap, oq=k + gap * 2 + 2 * 128 * 2) not in (BAD, UNSUPPORTED)   # behind the last row
