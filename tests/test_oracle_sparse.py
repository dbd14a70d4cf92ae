"""Pins of the sparse-attention and page-pool oracle: properties that follow from the definitions."""
import numpy as np
import pytest

from oracle import sparse_oracle as S
from oracle import wushkv_oracle as O


def _cache(rng, n, bits, d=128):
    K = rng.standard_normal((n, d)) * np.exp(0.5 * rng.standard_normal(d))
    codes, meta = [], []
    for k in K:
        c, step, low = O.quantize(k, bits, 0.96)
        codes.append(c)
        meta.append((step, low))
    return np.array(codes), np.array(meta)


@pytest.mark.parametrize("bits", [2, 3, 4])
def test_bounds_enclose_every_key_and_are_the_tightest_of_their_grid(bits):
    rng = np.random.default_rng(bits)
    codes, meta = _cache(rng, 37, bits)
    low, up, e = S.page_bounds(codes, meta)
    khat = np.float32(meta[:, 1:2] + meta[:, 0:1] * codes)
    assert np.all(low * 2.0 ** e <= khat.min(0)) and np.all(khat.max(0) <= up * 2.0 ** e)
    assert np.all((low + 1) * 2.0 ** e > khat.min(0)) and np.all(khat.max(0) > (up - 1) * 2.0 ** e)
    assert np.abs(np.stack([low, up])).max() <= 127 and np.abs(khat).max() > 127 * 2.0 ** (e - 1)
    zero = S.page_bounds(np.zeros((3, 128), int), np.zeros((3, 2)))
    assert not zero[0].any() and not zero[1].any() and zero[2] == -31


def test_scores_bound_the_logits_of_the_rounded_query():
    rng = np.random.default_rng(5)
    pages = [_cache(rng, 64, 2) for _ in range(6)]
    bounds = [S.page_bounds(*p) for p in pages]
    low, up, e = (np.stack([b[i] for b in bounds]) for i in range(3))
    for _ in range(5):
        q = rng.standard_normal(128) * 3
        qi, unit = S.fixed_point(q)
        assert np.abs(qi).max() == 32512 and np.abs(qi * unit - q).max() <= 0.5 * unit * (1 + 1e-12)
        s = S.page_scores(q, low, up, e, 0.1).astype(np.float64)
        for p, (codes, meta) in enumerate(pages):
            khat = np.float32(meta[:, 1:2] + meta[:, 0:1] * codes).astype(np.float64)
            # three roundings to 32 bits, relative to the score
            assert (khat @ (qi * unit) * float(np.float32(0.1))).max() <= s[p] + 4 * 2.0 ** -24 * abs(s[p])
    assert S.fixed_point(np.zeros(128))[1] == 0.0
    assert not S.fixed_point(np.full(128, np.inf))[0].any()


def test_selection_orders_by_key_then_index():
    keys = np.array([-3.0, 0.0, -1.0, -1.0, -np.inf, -1.0], dtype=np.float32)
    assert S.select(keys, 3).tolist() == [1, 2, 3]
    assert S.select(keys, 1, first=7).tolist() == [8]
    assert S.select(keys, 8).tolist() == [0, 1, 2, 3, 4, 5, -1, -1]
    # a sharp and a flat head: each head's best page has key 0
    low, up, e = -np.ones((2, 4), int), np.array([[100, 1, 1, 1], [1, 100, 1, 1]]), np.zeros(2, int)
    assert S.page_keys([np.array([50.0, 0, 0, 0]), np.array([0, 0.1, 0, 0])], low, up, e, 1.0).tolist() == [0.0, 0.0]


def test_all_pages_give_dense_attention_and_none_the_windows():
    rng = np.random.default_rng(9)
    n, s_sink, s_keep = 400, 4, 64
    K, V, q = rng.standard_normal((n, 128)), rng.standard_normal((n, 128)), rng.standard_normal(128)
    lo, hi, first, pages = S.packed_range(n, s_sink, s_keep, 1)
    assert (lo, hi, first, pages) == (4, 336, 0, 6)
    dense = O.attention_one_query(q, K, V, 0.1)
    np.testing.assert_allclose(S.sparse_attention(q, K, V, lo, hi, range(first, first + pages), 0.1), dense, rtol=1e-12)
    window = np.r_[0:4, 336:400]
    np.testing.assert_allclose(S.sparse_attention(q, K, V, lo, hi, [-1], 0.1), O.attention_one_query(q, K[window], V[window], 0.1), rtol=1e-12)
    assert S.packed_range(68, 4, 64, 1)[3] == 0 and S.packed_range(69, 4, 64, 1)[3] == 1


def test_pool_shares_copies_and_gives_back():
    p = S.Pool(4, 4, 6)
    assert p.reserve([(0, 0, 70)]) == [] and p.table[0].tolist() == [0, 1, -1, -1]
    p.fork(0, 1, 70)
    p.fork(0, 2, 70)
    assert p.refs.tolist() == [3, 3, 0, 0, 0, 0]
    # three holders of page 1 write: the last one keeps it
    assert p.reserve([(0, 70, 1), (1, 70, 1), (2, 70, 1)]) == [(1, 2), (1, 3)]
    assert p.table[:3, 1].tolist() == [2, 3, 1] and p.refs.tolist() == [3, 1, 1, 1, 0, 0]
    p.release(0)
    p.release(1, keep=64)
    assert p.table[1].tolist() == [0, -1, -1, -1] and p.refs.tolist() == [2, 1, 0, 0, 0, 0]
    p.fork(2, 0, 70)
    assert p.reserve([(3, 0, 256), (0, 70, 1)]) == [] and p.empty       # five pages wanted, four free: nothing is handed out
    assert p.table[0].tolist() == [0, -3, -1, -1] and p.table[3].tolist() == [-1] * 4
    p.check()
    assert p.reserve([(0, 70, 1)]) == [(1, 2)] and p.table[0, 1] == 2
    p.release(2)
    moves, live = p.compact()
    assert live == 2 and moves == [(2, 1)] and p.table[0].tolist() == [0, 1, -1, -1]
    p.check()


def test_pool_stays_consistent_over_random_calls():
    rng = np.random.default_rng(3)
    p, lens = S.Pool(6, 5, 17), [0] * 6
    for _ in range(400):
        a, b = (int(x) for x in rng.permutation(6)[:2])
        op = rng.integers(0, 4)
        if op == 0:
            new, before = int(rng.integers(0, 90)), p.table.copy()
            p.empty = False
            p.reserve([(a, lens[a], new)])
            if not p.empty and new and (lens[a] + new - 1) // 64 < 5:
                lens[a] += new
            else:
                assert np.array_equal(before >= 0, p.table >= 0) or p.empty
        elif op == 1 and all(e >= 0 for e in p.table[a, :-(-lens[a] // 64)]):
            p.fork(a, b, lens[a])
            lens[b] = lens[a]
        elif op == 2:
            lens[a] = int(rng.integers(0, lens[a] + 1))
            p.release(a, lens[a])
        else:
            p.compact()
        p.check()
