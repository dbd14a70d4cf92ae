"""The largest promised lengths: accepted up to the last one, with the list of a tight promise."""
import numpy as np
import pytest

from tests.test_abi_sparse_limits import WINDOWS, longest
from tests.test_gpu_sparse import Sparse, _close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_q,n_kv", [(4, 2), (8, 1)])
@pytest.mark.parametrize("s_sink,s_keep,s_flush,lag", WINDOWS)
def test_the_last_length_is_accepted(s_sink, s_keep, s_flush, lag, n_q, n_kv):
    s = Sparse([1400, 333], n_q, n_kv, 2, s_sink=s_sink, s_keep=s_keep, s_flush=s_flush, lag=lag, seed=31)
    q, Q = s.queries()
    tight_sel, _ = s.sparse(Q, 5)
    n = longest(s_sink, s_keep, s_flush, lag)
    sel, out = s.sparse(Q, 5, max_seq_len=n)
    assert np.array_equal(sel, tight_sel)
    for b in range(2):
        _close(out[b], s.oracle_attention(b, q[b], sel[b]))
    with pytest.raises(s.B.WushkvError):
        s.sparse(Q, 5, max_seq_len=n + 1)
    assert s.L.cache.status() == 0
