"""Sequences that go back without releasing the pages behind their length: what they write next is theirs alone.  Table, counts and
copy lists against the oracle; appends through two layers against caches that share nothing."""
import numpy as np
import pytest

from tests.test_gpu_page_pool import Pair, Server

pytestmark = pytest.mark.gpu


def owned(p, requests):
    """Every page that is about to be written is named by one entry."""
    table, refs = p.gpu.page_table.cpu().numpy(), p.gpu.refs.cpu().numpy()
    for slot, length, new in requests:
        pages = table[slot, length // 64:(length + new - 1) // 64 + 1] if new > 0 else []
        assert all(e >= 0 and refs[e] == 1 for e in pages)


def test_back_to_a_page_boundary_and_to_the_beginning():
    p = Pair(6, 8, 40)
    p.reserve([(0, 0, 195)])
    p.fork([0], [1], [195])
    back = [(0, 192, 1), (1, 192, 1)]                            # both at the boundary: the last keeps page 3
    assert p.reserve(back) == []
    owned(p, back)
    p.fork([0, 0], [2, 3], [193, 193])
    back = [(2, 0, 200), (3, 128, 1)]                            # a slot that is used anew, one that leaves the others at a whole page
    assert p.reserve(back) == []
    owned(p, back)
    p.fork([0, 0], [4, 5], [193, 193])
    back = [(4, 100, 60), (0, 128, 10), (5, 70, 200)]            # partly filled pages are copied, whole ones are not
    assert [c[0] for c in p.reserve(back)] == [int(p.ora.table[0, 1])] * 2
    owned(p, back)
    p.ora.check()


def test_all_holders_of_whole_and_partly_filled_pages():
    """The last holder keeps a page, whether it writes all of it or goes on in its middle."""
    for order in ([(0, 128, 3), (1, 130, 3)], [(1, 130, 3), (0, 128, 3)]):
        p = Pair(2, 4, 5)
        p.reserve([(0, 0, 131)])
        p.fork([0], [1], [131])
        assert len(p.reserve(order)) == (1 if order[0][0] == 1 else 0)
        owned(p, order)


def test_an_empty_pool_locks_whole_pages_too():
    p = Pair(3, 4, 4)
    p.reserve([(0, 0, 200)])
    p.fork([0], [1], [200])
    p.reserve([(1, 64, 100)])
    assert p.ora.empty and np.all(p.ora.table[1, 1:3] < -1) and p.ora.table[1, 3] >= 0
    p.reserve([(0, 0, 10), (2, 0, 1)])
    assert p.ora.empty and p.ora.table[0, 0] < -1
    p.release([0], [64])                                          # slot 0 keeps its first page: the others are slot 1's alone
    assert p.reserve([(1, 64, 100)]) == [] and p.ora.table[1].min() >= 0
    owned(p, [(1, 64, 100)])


@pytest.mark.parametrize("n_slots,max_pages,n_pages", [(2, 3, 7), (5, 4, 24), (16, 40, 700), (700, 5, 9000), (9, 300, 40000)])
def test_random_calls_with_lengths_that_go_back(n_slots, max_pages, n_pages):
    rng = np.random.default_rng(n_pages)
    p, lens, granted = Pair(n_slots, max_pages, n_pages), np.zeros(n_slots, int), 0
    for _ in range(24):
        op = rng.integers(0, 6)
        some = rng.permutation(n_slots)[:int(rng.integers(1, n_slots + 1))]
        if op <= 2:
            for s in some:                                        # to a length in the same page, to a boundary, to nothing
                kind = rng.integers(0, 4)
                lens[s] = [lens[s], lens[s] // 64 * 64, int(rng.integers(0, lens[s] + 1)), 0][kind]
            new = np.where(rng.random(len(some)) < 0.2, 0, rng.integers(1, 1 + 64 * max_pages // 3 + 1, len(some)))
            requests = [(int(s), int(lens[s]), int(n)) for s, n in zip(some, new)]
            p.reserve(requests)
            if not p.ora.empty:
                fit = [r for r in requests if r[1] + r[2] <= 64 * max_pages]
                owned(p, fit)
                granted += 1
                for s, length, n in fit:
                    lens[s] += n
        elif op <= 4 and n_slots > 1:
            half = len(some) // 2
            pairs = [(s, d) for s, d in zip(some[:half], some[half:]) if np.all(p.ora.table[s, :-(-lens[s] // 64)] != -1)]
            if pairs:
                src, dst = zip(*pairs)
                p.fork(src, dst, lens[list(src)])
                lens[list(dst)] = lens[list(src)]
        else:
            p.compact()
        p.ora.check()
    assert granted >= 3


@pytest.mark.parametrize("lengths,keepers", [((64, 70, 128), 0), ((64, 70), 1), ((70, 64, 64), 1)])
def test_many_holders_of_whole_pages(lengths, keepers):
    """More sequences than a tile of the ranking share their pages; where all of them write the second one, the last keeps it."""
    n = 1100
    p = Pair(n, 3, 3 * n, max_batch=n)
    p.reserve([(0, 0, 150)])
    p.fork([0] * (n - 1), list(range(1, n)), [150] * (n - 1))
    requests = [(int(s), lengths[s % len(lengths)], 30) for s in np.random.default_rng(2).permutation(n)]
    live = int((p.ora.refs > 0).sum())
    copies = p.reserve(requests)
    assert len(copies) == sum(r[1] == 70 for r in requests) - (keepers if requests[-1][1] == 70 else 0)
    assert int((p.ora.refs > 0).sum()) == live + n - keepers
    owned(p, requests)
    p.ora.check()


@pytest.mark.parametrize("bits", [2, 3, 4])
def test_rejected_draft_tokens_of_forked_sequences(bits):
    """A fork, both sides back to a boundary, appends to both: each reads its own tokens."""
    rng = np.random.default_rng(30 + bits)
    s = Server(5, 640, 40, bits=bits)
    s.append([0], [195], rng)
    s.fork([0, 0], [1, 2], rng)
    for slot in (0, 1):
        s.tokens[slot] = s.tokens[slot][:192]
    s.append([0, 1], [1, 1], rng)
    s.check(rng)
    s.append([1, 0, 2], [90, 3, 1], rng)
    s.check(rng)
    s.fork([1], [3], rng)
    s.tokens[3] = s.tokens[3][:64]
    s.tokens[1] = s.tokens[1][:130]
    s.append([3, 1], [300, 70], rng)
    s.check(rng)
    s.tokens[2] = []
    s.append([2], [150], rng)                                     # a slot that is used anew without a release
    s.check(rng)
    s.pool.compact(s.layers)
    s.check(rng)
