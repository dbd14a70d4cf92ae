"""Sequences whose tokens pass the table's end get nothing, and what a step does after the refused append leaves the pages that others
read further as they are."""
import numpy as np
import pytest

from tests.test_gpu_page_pool import Pair, Server

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_new", [127, 200])
def test_bounds_of_a_shared_page_stay_those_of_its_longest_sequence(n_new):
    torch, rng = pytest.importorskip("torch"), np.random.default_rng(n_new)
    s = Server(3, 256, 12)
    s.append([0], [195], rng)
    s.fork([0], [1], rng)
    s.pool.release(1, s.ints([1]), s.ints([130]))                  # page 2 is shared: 64 tokens of slot 0, two of slot 1
    s.tokens[1] = s.tokens[1][:130]
    before = [t.clone() for c in s.layers for t in (c.pages, c.bounds, c.exponents, c.ring_kv)]
    slots, lens, cu = s.ints([1]), s.ints([130]), s.ints([0, n_new])
    s.pool.reserve(s.layers, 1, slots, lens, cu)
    assert s.pool.status() == s.B.DEV_PAGE_TABLE_FULL
    s.pool.dev_status.zero_()
    for c in s.layers:
        K = torch.randn((n_new, 2, 128), device="cuda").to(torch.bfloat16).view(torch.int16)
        s.B.append(c.desc, 1, slots, lens, cu, n_new, n_new, K, K)
        s.B.update_page_bounds(c.desc, 1, slots, lens, cu, n_new, c.bounds, c.exponents)
        assert lens.tolist() == [130] and c.status() & s.B.DEV_PAGE_TABLE_FULL
        c.dev_status.zero_()
    for x, y in zip(before, [t for c in s.layers for t in (c.pages, c.bounds, c.exponents, c.ring_kv)]):
        assert torch.equal(x, y)
    s.append([1], [20], rng)                                       # a request that fits unlocks it
    s.check(rng)


def test_the_table_against_the_oracle():
    p = Pair(4, 4, 12)
    p.reserve([(0, 0, 195)])
    p.fork([0, 0], [1, 2], [195, 195])
    past = lambda *a: p.ora.reserve(list(a))  # noqa: E731
    for requests in ([(1, 130, 127), (2, 195, 1)], [(0, 192, 65), (1, 250, 7)], [(2, 300, 5), (1, 256, 1)], [(3, 10, 500)]):
        copies = past(*requests)
        slots, lens, new = zip(*requests)
        p.gpu.reserve([], len(requests), p.ints(slots), p.ints(lens), p.ints(np.concatenate([[0], np.cumsum(new)])))
        p.check(copies, len(requests))
        assert p.gpu.status() == p.B.DEV_PAGE_TABLE_FULL
        p.gpu.dev_status.zero_()
    assert p.ora.table[1, 2] < -1 and p.ora.table[1, 3] < -1
    p.reserve([(1, 130, 100)])
    assert p.ora.table[1].min() >= 0
