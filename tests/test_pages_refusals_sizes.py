"""Sizes at which the paged-cache calls would count beyond their integers: refused on the host (the addresses are never dereferenced)."""
import ctypes as C

import pytest

from paper_2601_20357_b200 import binding as B
from test_pages_refusals import pages, query


@pytest.mark.parametrize("tokens,heads,refused", [(0x7FFFFFF0, 2, True), (0x7FFFFF80, 2, True), (0x7FFFFF01, 2, True), (0x3FFFFFC0, 4, True), (0x7FFFFF00, 2, False),
                                                  (0x3FFFFF80, 4, False)])
def test_attention_counts_query_rows_up_to_the_end_of_a_tile(tokens, heads, refused):
    """Rows a KV head (tokens times heads / 2): the last tile of 256 may end 255 behind them.  What is not refused goes on to the device, which is not there."""
    t = query(n_tokens=tokens, max_new=tokens, n_heads=heads)
    assert B.lib().tabed_pages_attention(C.byref(pages()), C.byref(t)) == (B.ERR_UNSUPPORTED if refused else B.ERR_CUDA)
