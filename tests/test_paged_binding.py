"""Sizes and arguments of the calls over a paged cache, on the host."""
import pytest

from paper_2506_19645_amd import binding as B


@pytest.mark.parametrize("T,heads,kv", [(8, 32, 32), (8, 64, 8), (4, 32, 8), (1, 40, 1), (1, 8, 8), (2, 6, 2)])
def test_one_workspace_serves_smaller_batches(T, heads, kv):
    """Sized for the most new tokens, whatever the rows, the sequences and the table: no call with fewer of any is refused."""
    last = 0
    for max_new in (1, 2, 3, 4, 5, 8, 9, 16, 17, 32, 33, 64, 65, 500, 2048, 8192):
        sizes = {B.paged_attn_workspace_bytes(B.paged_desc(T=T, batch=batch, n_heads=heads, n_kv_heads=kv, rows=rows, max_new=max_new,
                                                           page_size=16, n_pages=1 << 20, max_pages=columns, cache_type=cache))
                 for batch in (1, 3, 64, 1000) for rows in (1, 8, 100, 1536, 4096, 20000) for columns in (1, 64, 8192)
                 for cache in (B.CACHE_BF16, B.CACHE_E4M3)}
        assert len(sizes) == 1
        size = sizes.pop()
        assert size >= last and size > 0
        last = size
