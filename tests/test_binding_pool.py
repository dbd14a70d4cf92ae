"""Combinations of arguments that PagedCache and PagePool refuse (no GPU needed)."""
import numpy as np
import pytest

from paper_2609_38121_b200 import binding as B

T = np.eye(128, dtype=np.float32)[None]


def test_a_cache_in_a_pool_has_no_page_order_of_its_own():
    pool = B.PagePool(2, 256, 8, device="cpu")
    make = lambda **kw: B.PagedCache(2, 1, 2, 2, 256, 4, 64, 1, 0.96, 0.92, T, T, device="cpu", **kw)  # noqa: E731
    assert make(pool=pool).page_table is pool.page_table
    assert make(page_order=np.arange(8)[::-1]).page_table.tolist() == [[7, 6, 5, 4], [3, 2, 1, 0]]
    with pytest.raises(ValueError):
        make(pool=pool, page_order=np.arange(8))
    with pytest.raises(ValueError):
        B.PagedCache(2, 1, 2, 3, 256, 4, 64, 1, 0.96, 0.92, T, T, device="cpu", pool=pool)
