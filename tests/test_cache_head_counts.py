"""Calls whose sequences cannot be counted in 31 bits are refused: before anything is enqueued,
so without a GPU. No pointer here is dereferenced."""
import pytest

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300 import _lib as L

FAKE = 1 << 40


def _shape(heads, batch):
    return M.make_shape(heads, heads, 64, 2, 0, [0] * batch + [1], [1] * batch)


@pytest.mark.parametrize("heads,batch,ok", [(2 ** 24, 64, True), (2 ** 24 + 1, 64, False), (2 ** 26, 64, False),
                                            (2 ** 30, 1, True), (2 ** 30, 2, False)])
def test_sequences_past_31_bits(heads, batch, ok):
    s = _shape(heads, batch)
    c = L.Cache(dtype=0, page_size=32, n_pages=100, max_pages=9, k_pages=FAKE, v_pages=FAKE, page_table=FAKE, lens=FAKE)
    if ok:
        assert M.mmshift_cache_workspace_size(s, c) > 256
        return
    with pytest.raises(M.MMShiftError) as e:
        M.mmshift_cache_workspace_size(s, c)
    assert e.value.code == L.MMSHIFT_ERR_UNSUPPORTED
    n = 1 << 40
    assert [M.mmshift_cache_append(s, c, FAKE, FAKE, 0, FAKE, n), M.mmshift_cache_read(s, c, None, FAKE, FAKE, FAKE, n),
            M.mmshift_cache_attention(s, c, FAKE, 0, 1, 0.0, FAKE, None, FAKE, n)] == [L.MMSHIFT_ERR_UNSUPPORTED] * 3
