"""Sparse attention by its other forms, all against the oracle: the list handed back to the call that takes one, CTAs of four warps
at every bit width and with every input, rows of one sequence at several lengths."""
import numpy as np
import pytest

from oracle import sparse_oracle as S
from oracle import wushkv_oracle as O
from paper_2609_38121_b200 import workloads as W
from tests.test_gpu_sparse import SCALE, Sparse, _close

pytestmark = pytest.mark.gpu

LENGTHS = [1500, 0, 1, 68, 69, 333, 2050]


@pytest.fixture
def four_warps():
    from paper_2609_38121_b200 import binding as B
    B.set_test_option("select_cluster", -1)
    yield
    B.set_test_option("select_cluster", 0)


def _check_list_form(s, n_select):
    """The outputs of a selected list that is handed over again."""
    q, Q = s.queries()
    sel, _ = s.sparse(Q, n_select)
    assert np.array_equal(sel, s.oracle_select(q, n_select))
    for b in range(s.L.batch):
        if s.L.done[b] == 0:
            assert not s.by_list[b].any()
        else:
            _close(s.by_list[b], s.oracle_attention(b, q[b], sel[b]))
    assert s.L.cache.status() == 0


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("n_q,n_kv", [(6, 2), (8, 2), (5, 1), (16, 2)])
def test_the_selected_list_handed_over(bits, n_q, n_kv):
    _check_list_form(Sparse(LENGTHS, n_q, n_kv, bits, seed=40 + bits), 5)


def test_long_lists_handed_over():
    _check_list_form(Sparse([45000, 36000], 4, 1, 2, seed=44), 560)


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (6, 2), (8, 2)])
def test_ctas_of_four_warps(four_warps, bits, n_q, n_kv):
    s = Sparse(LENGTHS, n_q, n_kv, bits, seed=50 + bits)
    s.check(5)
    s.check(40)
    _check_list_form(s, 7)


@pytest.mark.parametrize("bits", [2, 3])
@pytest.mark.parametrize("s_sink,s_keep,s_flush,lag", [(0, 64, 1, 0), (130, 64, 8, 0), (4, 128, 1, 3)])
def test_ctas_of_four_warps_with_other_windows(four_warps, bits, s_sink, s_keep, s_flush, lag):
    Sparse([1111, 129, 211, 64 + s_sink], s_sink=s_sink, s_keep=s_keep, s_flush=s_flush, lag=lag, seed=60, n_q=6, n_kv=2, bits=bits).check(4)


@pytest.mark.parametrize("bits", [2, 3, 4])
def test_ctas_of_four_warps_on_lists_of_the_caller(four_warps, bits):
    s = Sparse([1500, 400, 1000], 6, 2, bits, seed=61)
    q, Q = s.queries()
    lists = np.full((3, 2, 7), -1)
    lists[0, 0], lists[0, 1] = [20, -1, 3, 0, 22, -1, 11], [5, 4, 3, 2, 1, 0, -1]
    lists[1, 0, :5], lists[1, 1, :5] = [5, 4, -1, 0, 1], [-1, -1, -1, -1, 2]
    _, out = s.sparse(Q, 7, selected=lists)
    for b in range(3):
        _close(out[b], s.oracle_attention(b, q[b], lists[b]))
    assert s.L.cache.status() == 0


@pytest.mark.parametrize("bits", [2, 4])
def test_ctas_of_four_warps_with_projected_queries(four_warps, bits):
    """Against the oracle's attention of the prepared queries, over the kernel's own list."""
    from tests.test_gpu_projected import EPS, _prepared
    s = Sparse([1500, 800], 8, 2, bits, seed=62, rmsnorm=True)
    qp = np.stack([s.wl.projected(b, s.L.done[b])[1][-1] for b in range(2)])
    pro = s.B.Prologue(s.wl.theta, 2048, normalise=True, q_weight=s.wl.gain_q, eps=EPS)
    Q = s.torch.from_numpy(W.f32_to_bf16_bits(qp.astype(np.float32)).view(np.int16)).cuda()
    sel, out = s.sparse(Q, 4, prologue=pro.desc)
    checked = 0
    for b in range(2):
        y, doubtful = _prepared(W.bf16_round_f32(qp.astype(np.float32))[b][None], np.array([s.L.done[b] - 1]), s.wl.theta, s.wl.gain_q[None], True)
        ref = s.oracle_attention(b, y[0], sel[b])
        for h in range(2):
            if not doubtful[0][4 * h:4 * h + 4].any():
                _close(out[b, 4 * h:4 * h + 4], ref[4 * h:4 * h + 4])
                _close(s.by_list[b, 4 * h:4 * h + 4], ref[4 * h:4 * h + 4])
                checked += 1
    assert checked >= 2 and s.L.cache.status() == 0


@pytest.mark.parametrize("cluster", [0, -1, 1, 4])
def test_rows_of_one_sequence_select_like_sequences_of_their_lengths(cluster):
    s = Sparse([1300, 500], 8, 2, 2, seed=63, ring_cap=80)
    rows = [(0, 1300), (0, 1299), (0, 1290), (1, 500), (0, 1297), (1, 487)]
    ints = lambda k: s.torch.tensor([r[k] for r in rows], dtype=s.torch.int32, device="cuda")  # noqa: E731
    q = np.stack([s.wl.queries(b, n - 1) for b, n in rows])
    Q = s.torch.from_numpy(W.f32_to_bf16_bits(q).view(np.int16)).cuda()
    s.B.set_test_option("select_cluster", cluster)
    try:
        sel, out = s.sparse(Q, 4, batch=len(rows), slot=ints(0), seq_len=ints(1))
    finally:
        s.B.set_test_option("select_cluster", 0)
    for r, (b, n) in enumerate(rows):
        _, _, first, pages = S.packed_range(n, 4, 64, 1)
        for h in range(2):
            # bounds are those of all tokens in the pages, also of those behind the row's length
            low, up, e = (x[first:first + pages] for x in s.oracle_bounds(b, h))
            qc = [O.query_compensation(s.L.TinvT[h].astype(np.float32), q[r, 4 * h + g][None])[0] for g in range(4)]
            assert np.array_equal(sel[r, h], S.select(S.page_keys(qc, low, up, e, SCALE), 4, first))
        _close(out[r], s.oracle_attention(b, q[r], sel[r], length=n))
    assert s.L.cache.status() == 0
