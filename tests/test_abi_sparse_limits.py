"""The longest sequences that page selection accepts: 16384 packed pages, at the first length beyond them a refusal (no GPU needed)."""
import pytest

from oracle import sparse_oracle as S
from paper_2609_38121_b200 import binding as B
from tests.test_abi_sparse import BOUNDS, SELECT, SPARSE, _cache

WINDOWS = [(4, 64, 1, 0), (0, 1, 1, 0), (130, 64, 8, 0), (4, 128, 1, 3), (4, 32, 16, 0)]


def longest(s_sink, s_keep, s_flush, lag):
    """The largest number of positions with at most 16384 packed pages."""
    n = 1 << 20
    while S.packed_range(n + 1, s_sink, s_keep, s_flush, lag)[3] <= 16384:
        n += 1
    return n


@pytest.mark.parametrize("s_sink,s_keep,s_flush,lag", WINDOWS)
def test_the_first_length_beyond_is_refused(s_sink, s_keep, s_flush, lag):
    n = longest(s_sink, s_keep, s_flush, lag)
    assert S.packed_range(1 << 20, s_sink, s_keep, s_flush, lag)[3] <= 16384 and n >= 1 << 20
    cache = _cache(s_sink=s_sink, s_keep=s_keep, s_flush=s_flush, boundary_lag=lag, ring_cap=s_keep + s_flush - 1 + lag)
    for fn, args in ((B.lib.wushkv_select_pages, SELECT), (B.lib.wushkv_decode_attn_sparse, SPARSE)):
        for length in (n + 1, n + 64, (1 << 31) - 1):
            assert fn(*{**args, "cache": cache, "max_seq_len": length}.values(), None) == B.ECAPACITY, length


def test_more_bounds_than_a_grid_holds_are_refused():
    huge = _cache(n_q=65535, n_kv=65535, max_pages=1 << 20)
    assert B.lib.wushkv_update_page_bounds(*{**BOUNDS, "cache": huge, "max_new": 1 << 30}.values(), None) == B.ECAPACITY
