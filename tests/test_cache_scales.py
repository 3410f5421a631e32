"""Softmax scales that base 2 cannot take are refused before anything is enqueued, so without
a GPU. No pointer here is dereferenced."""
import pytest

import paper_2607_22586_gb300 as M
from paper_2607_22586_gb300 import _lib as L

FAKE = 1 << 40


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_past_float32_in_base_2(scale):
    """scale * log2(e) is above float32's largest: every logit would be a NaN or an infinity."""
    s = M.make_shape(8, 2, 128, 2, 0, [0, 3], [1])
    c = L.Cache(dtype=0, page_size=32, n_pages=100, max_pages=9, k_pages=FAKE, v_pages=FAKE, page_table=FAKE, lens=FAKE)
    assert M.mmshift_cache_attention(s, c, FAKE, 0, 1, scale, FAKE, None, FAKE, 1 << 40) == L.MMSHIFT_ERR_INVALID_ARG
