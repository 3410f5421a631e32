"""Refusals of the calls on a pool's pages and of attention in groups: before anything is
enqueued, so without a GPU. No pointer here is dereferenced."""
import pytest
import torch

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300 import _lib as L
from paper_2607_22586_gb300.cache import PagedKVCache
from tests.test_cache_abi import FAKE, _cache, _shape

BAD, UNSUPPORTED, WORKSPACE = L.MMSHIFT_ERR_INVALID_ARG, L.MMSHIFT_ERR_UNSUPPORTED, L.MMSHIFT_ERR_WORKSPACE
BIG = 1 << 40


def _calls(s, c, refs=FAKE, ws=FAKE, n=BIG):
    return [M.mmshift_cache_reserve(s, c, refs, ws, n), M.mmshift_cache_fork(s, c, refs, [0], [1], ws, n),
            M.mmshift_cache_free(s, c, refs, [0, 2], ws, n), M.mmshift_cache_compact(s, c, refs, FAKE, None, ws, n)]


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=1), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(n_pages=0), BAD), (dict(lens=None), BAD),
    (dict(page_table=None), BAD), (dict(dtype=2), BAD), (dict(k_pages=FAKE + 8), BAD),
])
def test_bad_caches(bad, code):
    s, c = _shape(), _cache(**bad)
    assert _calls(s, c) == [code] * 4
    assert M.mmshift_cache_attention_shared(s, c, [0, 3], FAKE, 0, 1, 0.0, FAKE, None, FAKE, BIG) == code
    for size in (lambda: M.mmshift_cache_pages_workspace_size(s, c),
                 lambda: M.mmshift_cache_shared_workspace_size(s, c, [0, 3])):
        with pytest.raises(M.MMShiftError) as e:
            size()
        assert e.value.code == code


def test_bad_counts_and_workspaces():
    s, c = _shape(), _cache()
    assert _calls(s, c, refs=None) == [BAD] * 4
    assert _calls(s, c, refs=FAKE + 2) == [BAD] * 4
    assert _calls(s, c, ws=None) == [WORKSPACE] * 4
    assert _calls(s, c, ws=FAKE + 8) == [WORKSPACE] * 4
    assert _calls(s, c, n=255) == [WORKSPACE] * 4
    n = M.mmshift_cache_pages_workspace_size(s, c)
    assert _calls(s, c, n=n - 1)[0] == _calls(s, c, n=n - 1)[3] == WORKSPACE


@pytest.mark.parametrize("src,dst", [([0], [0]), ([0], [3]), ([0], [-1]), ([3], [0]), ([-1], [0]), ([0, 0], [1, 1]),
                                     ([0, 1], [1, 2]), ([0, 1], [2, 0])])
def test_bad_forks(src, dst):
    assert M.mmshift_cache_fork(_shape(), _cache(), FAKE, src, dst, FAKE, BIG) == BAD


def test_bad_lists():
    s, c = _shape(), _cache()
    for which in ([0, 0], [3], [-1], [0, 1, 2, 0]):
        assert M.mmshift_cache_free(s, c, FAKE, which, FAKE, BIG) == BAD
    lib, byref = M.load_library(), M._lib.ctypes.byref
    assert lib.mmshift_cache_fork(byref(s), byref(c), FAKE, 1, None, L._ints([1]), FAKE, BIG, None) == BAD
    assert lib.mmshift_cache_fork(byref(s), byref(c), FAKE, 1, L._ints([1]), None, FAKE, BIG, None) == BAD
    assert lib.mmshift_cache_free(byref(s), byref(c), FAKE, 1, None, FAKE, BIG, None) == BAD
    assert lib.mmshift_cache_free(byref(s), byref(c), FAKE, -1, L._ints([1]), FAKE, BIG, None) == BAD
    assert M.mmshift_cache_compact(s, c, FAKE, None, None, FAKE, BIG) == BAD
    assert M.mmshift_cache_compact(s, c, FAKE, FAKE + 1, None, FAKE, BIG) == BAD
    assert M.mmshift_cache_compact(s, c, FAKE, FAKE, FAKE + 2, FAKE, BIG) == BAD


def test_nothing_to_do_is_no_error():
    s, c = _shape(cu_seqlens=[0, 0, 0, 0]), _cache()
    assert M.mmshift_cache_reserve(s, c, FAKE, FAKE, BIG) == L.MMSHIFT_OK
    assert M.mmshift_cache_compact(s, c, FAKE, None, None, FAKE, BIG) == L.MMSHIFT_OK
    assert M.mmshift_cache_fork(s, c, FAKE, [], [], FAKE, BIG) == L.MMSHIFT_OK
    assert M.mmshift_cache_free(s, c, FAKE, [], FAKE, BIG) == L.MMSHIFT_OK
    assert M.mmshift_cache_attention_shared(s, c, [0, 3], None, 0, 1, 0.0, None, None, FAKE, BIG) == L.MMSHIFT_OK


@pytest.mark.parametrize("groups", [[0], [0, 2], [0, 4], [1, 3], [0, 1, 1, 3], [0, 2, 1, 3], [0, 1, 2, 3, 3]])
def test_bad_groups(groups):
    s, c = _shape(), _cache()
    assert M.mmshift_cache_attention_shared(s, c, groups, FAKE, 0, 1, 0.0, FAKE, None, FAKE, BIG) == BAD
    with pytest.raises(M.MMShiftError) as e:
        M.mmshift_cache_shared_workspace_size(s, c, groups)
    assert e.value.code == BAD


@pytest.mark.parametrize("bad,code", [
    (dict(q=None), BAD), (dict(q=FAKE + 1), BAD), (dict(out=None), BAD), (dict(out=FAKE + 1), BAD), (dict(lse=FAKE + 1), BAD),
    (dict(stride=8), BAD), (dict(causal=-1), BAD), (dict(scale=-0.5), BAD), (dict(scale=float("inf")), BAD),
    (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 16), WORKSPACE), (dict(n=4096), WORKSPACE), (dict(layers=2), UNSUPPORTED),
])
def test_bad_shared_arguments(bad, code):
    a = dict(q=FAKE, stride=0, causal=1, scale=0.0, out=FAKE, lse=None, ws=FAKE, n=BIG, layers=1)
    a.update(bad)
    s = _shape(n_layers=a["layers"])
    assert M.mmshift_cache_attention_shared(s, _cache(), [0, 2, 3], a["q"], a["stride"], a["causal"], a["scale"], a["out"],
                                            a["lse"], a["ws"], a["n"]) == code


def test_more_sequences_than_blocks_count():
    s = _shape(n_q_heads=2 ** 27, n_kv_heads=2 ** 27, cu_seqlens=[0, 1, 1, 2])
    assert M.mmshift_cache_attention_shared(s, _cache(), [0, 3], FAKE, 0, 1, 0.0, FAKE, None, FAKE, BIG) == UNSUPPORTED
    with pytest.raises(M.MMShiftError) as e:
        M.mmshift_cache_shared_workspace_size(s, _cache(), [0, 3])
    assert e.value.code == UNSUPPORTED


def test_the_class_refuses():
    make = lambda **kw: PagedKVCache(**{**dict(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, batch=3,  # noqa: E731
                                               rows=40, page_size=16, device="cpu"), **kw})
    with pytest.raises(ValueError):
        make(pages=0)
    with pytest.raises(ValueError):
        make(pages=10, rows=torch.tensor([[[40, 41]] * 3]))
    own = make()
    for bad in (lambda: own.fork([0], [1]), lambda: own.free([0]), lambda: own.compact(torch.zeros(1, 3, 2, dtype=torch.int32), [1] * 3)):
        with pytest.raises((ValueError, AssertionError, RuntimeError)):
            bad()
    pool = make(pages=7)
    assert pool.k_pages.shape[0] == 7 and not pool.refs.any() and (pool.page_table == -1).all() and pool.capacity == 48
