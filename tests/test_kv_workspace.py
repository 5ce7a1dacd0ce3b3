"""Workspace of the cache's attention: it is for partial sums of what is cut, not
for every row that an entry might have (no GPU needed)."""
import ctypes

import pytest

from paper_2606_00021_amd import sense
from test_kv_abi import cache


def size(n, max_rows, n_heads, max_kv=0, **kw):
    out = ctypes.c_size_t()
    c = cache(n_kv_heads=8, head_dim=128, page_size=32, max_pages=1024, n_seqs=8192, **kw)
    assert sense.load_library().sense_kv_attention_workspace_size(
        ctypes.byref(c), n, max_rows, n_heads, max_kv, ctypes.byref(out)) == 0
    return out.value


@pytest.mark.parametrize("n", [64, 256, 1000])
def test_tokens_beside_a_long_chunk(n):
    """2048 rows for one entry of n: 2.2 GB and more if every entry had room."""
    assert 0 < size(n, 2048, 32) < 150 << 20


def test_more_entries_or_rows_never_need_less():
    for heads in (8, 32, 64):
        last = 0
        for n in (1, 2, 8, 63, 64, 65, 200, 1000):
            now = size(n, 1, heads)
            assert now >= last
            last = now
    assert size(64, 2048, 32, max_kv=1024) == 0
