"""Refusals of the paged cache's entry points: before anything is enqueued, so
without a GPU. No pointer here is dereferenced."""
import ctypes

import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300 import _lib as L

FAKE = 1 << 40


def _shape(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, window=2, dtype=0, cu_seqlens=[0, 3, 3, 10],
                budgets=[4, 1, 2])
    base.update(kw)
    return M.make_shape(**base)


def _cache(**kw):
    base = dict(dtype=0, page_size=32, n_pages=100, max_pages=9, k_pages=FAKE, v_pages=FAKE, k_scales=None,
                v_scales=None, page_table=FAKE, lens=FAKE)
    base.update(kw)
    return L.Cache(**base)


def _calls(s, c, ws=FAKE, n=None, Q=FAKE, K=FAKE, out=FAKE, stride=0):
    """Statuses of append, read and attention."""
    n = 1 << 40 if n is None else n
    return [M.mmshift_cache_append(s, c, K, FAKE, stride, ws, n),
            M.mmshift_cache_read(s, c, None, out, FAKE, ws, n),
            M.mmshift_cache_attention(s, c, Q, stride, 1, 0.0, out, None, ws, n)]


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=1), L.MMSHIFT_ERR_UNSUPPORTED),                 # float32 pages of a bfloat16 call
    (dict(dtype=3), L.MMSHIFT_ERR_UNSUPPORTED),
    (dict(page_size=8), L.MMSHIFT_ERR_UNSUPPORTED),
    (dict(page_size=48), L.MMSHIFT_ERR_UNSUPPORTED),
    (dict(page_size=512), L.MMSHIFT_ERR_UNSUPPORTED),
    (dict(n_pages=0), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(n_pages=2 ** 26), L.MMSHIFT_ERR_UNSUPPORTED),         # rows past 31 bits
    (dict(max_pages=0), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(max_pages=2 ** 26), L.MMSHIFT_ERR_UNSUPPORTED),
    (dict(k_pages=None), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(v_pages=FAKE + 8), L.MMSHIFT_ERR_INVALID_ARG),        # unaligned
    (dict(page_table=None), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(page_table=FAKE + 2), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(lens=None), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(dtype=2), L.MMSHIFT_ERR_INVALID_ARG),                 # 8-bit pages without scales
    (dict(dtype=2, k_scales=FAKE, v_scales=FAKE + 2), L.MMSHIFT_ERR_INVALID_ARG),
])
def test_bad_caches(bad, code):
    s, c = _shape(), _cache(**bad)
    assert _calls(s, c) == [code] * 3
    full = _shape(cu_seqlens=[0, 3, 5, 10])
    assert M.mmshift_cache_fill(full, c, FAKE, FAKE, FAKE, None, FAKE, 256) == code
    with pytest.raises(M.MMShiftError) as e:
        M.mmshift_cache_workspace_size(s, c)
    assert e.value.code == code


@pytest.mark.parametrize("bad,code", [
    (dict(n_q_heads=7), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(head_dim=96), L.MMSHIFT_ERR_UNSUPPORTED),
    (dict(dtype=2), L.MMSHIFT_ERR_UNSUPPORTED),
    (dict(cu_seqlens=[0, 3, 2, 10]), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(cu_seqlens=[1, 3, 4, 10]), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(cu_seqlens=[0, 3, 4, 2 ** 30]), L.MMSHIFT_ERR_UNSUPPORTED),
    (dict(cu_seqlens=list(range(66)), budgets=[1] * 65), L.MMSHIFT_ERR_INVALID_ARG),
    (dict(n_layers=0), L.MMSHIFT_ERR_INVALID_ARG),
])
def test_bad_shapes(bad, code):
    assert _calls(_shape(**bad), _cache()) == [code] * 3


def test_bad_arguments():
    s, c = _shape(), _cache()
    n = M.mmshift_cache_workspace_size(s, c)
    assert n >= 256
    assert _calls(s, c, ws=None) == _calls(s, c, ws=FAKE + 16) == [L.MMSHIFT_ERR_WORKSPACE] * 3
    assert _calls(s, c, n=255) == [L.MMSHIFT_ERR_WORKSPACE] * 3
    assert _calls(s, c, n=n - 1)[2] == L.MMSHIFT_ERR_WORKSPACE
    assert _calls(s, c, Q=None, K=None, out=None) == [L.MMSHIFT_ERR_INVALID_ARG] * 3
    assert _calls(s, c, Q=FAKE + 1, K=FAKE + 1, out=FAKE + 1) == [L.MMSHIFT_ERR_INVALID_ARG] * 3
    for stride in (-1, 255):                                     # rows that overlap
        got = _calls(s, c, stride=stride)
        assert got[0] == got[2] == L.MMSHIFT_ERR_INVALID_ARG
    for causal, scale in ((2, 0.0), (-1, 0.0), (1, -1.0), (1, float("nan")), (0, float("inf"))):
        assert M.mmshift_cache_attention(s, c, FAKE, 0, causal, scale, FAKE, None, FAKE, n) == L.MMSHIFT_ERR_INVALID_ARG
    assert M.mmshift_cache_attention(s, c, FAKE, 0, 1, 0.0, FAKE, FAKE + 2, FAKE, n) == L.MMSHIFT_ERR_INVALID_ARG
    assert M.mmshift_cache_read(s, c, FAKE + 1, FAKE, FAKE, FAKE, n) == L.MMSHIFT_ERR_INVALID_ARG
    two = _shape(n_layers=2, layer_stride_kv=10 * 2 * 128 - 1, layer_stride_q=1 << 20)
    n = M.mmshift_cache_workspace_size(two, c)
    assert M.mmshift_cache_append(two, c, FAKE, FAKE, 0, FAKE, n) == L.MMSHIFT_ERR_INVALID_ARG
    assert M.mmshift_cache_attention(two, c, FAKE, 0, 1, 0.0, FAKE, None, FAKE, n) == L.MMSHIFT_ERR_UNSUPPORTED
    # fill: a prompt has no empty request, and its keys are no pageable host memory
    assert M.mmshift_cache_fill(s, c, FAKE, FAKE, FAKE, None, FAKE, n) == L.MMSHIFT_ERR_INVALID_ARG
    full = _shape(cu_seqlens=[0, 3, 5, 10])
    assert M.mmshift_cache_fill(full, c, FAKE, FAKE, None, None, FAKE, n) == L.MMSHIFT_ERR_INVALID_ARG
    assert M.mmshift_cache_fill(full, c, FAKE, FAKE, FAKE, FAKE + 2, FAKE, n) == L.MMSHIFT_ERR_INVALID_ARG
    assert M.mmshift_cache_fill(full, c, FAKE, FAKE, FAKE, None, FAKE, 255) == L.MMSHIFT_ERR_WORKSPACE


def test_calls_without_rows_do_nothing():
    s, c = _shape(cu_seqlens=[0, 0, 0, 0]), _cache()
    n = M.mmshift_cache_workspace_size(s, c)
    assert _calls(s, c, n=n) == [L.MMSHIFT_OK] * 3
    assert _calls(s, c, n=n, Q=None, K=None, out=None) == [L.MMSHIFT_OK] * 3


def test_make_cache_refuses_what_the_library_cannot_see():
    pages, table, lens = torch.zeros(4, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int32), \
        torch.zeros(2, dtype=torch.int32)
    c = M.make_cache(pages, pages.clone(), table, lens)
    assert (c.page_size, c.n_pages, c.max_pages, c.dtype) == (16, 4, 2, L.MMSHIFT_BF16)
    codes, scales = torch.zeros(4, 16, 64, dtype=torch.int8), torch.zeros(4, 16)
    assert M.make_cache(codes, codes, table, lens, scales, scales).dtype == L.MMSHIFT_I8
    for args in ((pages, pages[:3], table, lens), (pages.half(), pages.half(), table, lens),
                 (pages, pages.float(), table, lens), (pages, pages, table.long(), lens),
                 (pages, pages, table, lens[:1]), (pages, pages.transpose(1, 2).contiguous().transpose(1, 2), table, lens),
                 (codes, codes, table, lens), (codes, codes, table, lens, scales, scales[:, :8]),
                 (pages, pages, table, lens, scales, scales)):
        with pytest.raises(ValueError):
            M.make_cache(*args)


def test_struct_layout_is_c():
    assert ctypes.sizeof(L.Cache) == 4 * 4 + 6 * 8
