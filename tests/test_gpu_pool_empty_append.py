"""Appends of several tokens after a reserve that an empty pool refused: the sequence goes on reading what it had, with the window at
the smallest ring, and takes the same tokens once there is room."""
import numpy as np
import pytest

from tests.test_gpu_page_pool import Server

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("n_new", [2, 4, 70, 140])
def test_a_refused_step_leaves_the_sequence_as_it_was(bits, n_new):
    torch, rng = pytest.importorskip("torch"), np.random.default_rng(n_new)
    s = Server(4, 320, 7, bits=bits)
    s.append([0, 1], [126, 100], rng)
    s.fork([1], [2], rng)                                          # its last page is shared: locked where the pool is empty
    s.append([3], [192], rng)                                      # the pool is full
    before = [t.clone() for c in s.layers for t in (c.pages, c.ring_kv, c.sink_kv)]
    slots, lens, counts = [0, 2, 1], [126, 100, 100], [n_new + 1, n_new, n_new]
    cu = s.ints(np.concatenate([[0], np.cumsum(counts)]))
    s.pool.reserve(s.layers, 3, s.ints(slots), s.ints(lens), cu)
    assert s.pool.status() == s.B.DEV_POOL_EMPTY
    for c in s.layers:
        seq_len = s.ints(lens)
        K, V = (torch.randn((sum(counts), 2, 128), device="cuda").to(torch.bfloat16).view(torch.int16) for _ in range(2))
        s.B.append(c.desc, 3, s.ints(slots), seq_len, cu, sum(counts), max(counts), K, V)
        s.B.update_page_bounds(c.desc, 1, s.ints([0]), seq_len, cu, max(counts), c.bounds, c.exponents)
        assert seq_len.tolist() == lens and c.status() == s.B.DEV_BAD_PAGE_ID
        c.dev_status.zero_()
    for x, y in zip(before, [t for c in s.layers for t in (c.pages, c.ring_kv, c.sink_kv)]):
        assert torch.equal(x, y)
    s.pool.dev_status.zero_()
    table, saved = s.pool.page_table, s.pool.page_table.clone()
    assert int((table < -1).sum()) == 2                            # both holders of the shared page; its entries count as they are
    table.copy_(torch.where(table < -1, -2 - table, table))
    s.check(rng)
    table.copy_(saved)
    s.release([3])
    s.append([0, 2, 1], [min(n_new + 1, 60), 3, 2], rng)
    s.check(rng)
