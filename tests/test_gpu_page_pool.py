"""The page pool on the GPU against the oracle that carries the same calls out one request after the other: table, counts and
copy lists are equal number by number; copies of pages and windows; sequences that share pages behave like sequences of their own."""
import numpy as np
import pytest

from oracle import sparse_oracle as S
from paper_2609_38121_b200 import workloads as W
from tests.harness import oracle_transforms

pytestmark = pytest.mark.gpu


class Pair:
    """A pool on both sides."""

    def __init__(self, n_slots, max_pages, n_pages, max_batch=None):
        import torch
        from paper_2609_38121_b200 import binding as B
        self.torch, self.B = torch, B
        self.gpu = B.PagePool(n_slots, 64 * max_pages, n_pages, max_batch=max_batch or n_slots)
        self.ora = S.Pool(n_slots, max_pages, n_pages)

    def ints(self, values):
        return self.torch.tensor([int(v) for v in values], dtype=self.torch.int32, device="cuda")

    def check(self, copies=None, capacity=None):
        assert np.array_equal(self.gpu.page_table.cpu().numpy(), self.ora.table)
        assert np.array_equal(self.gpu.refs.cpu().numpy(), self.ora.refs)
        if copies is not None:
            got = self.gpu.copies[:, :capacity].cpu().numpy()
            assert int(self.gpu.n_copies.item()) == len(copies)
            assert [tuple(x) for x in got.T[:len(copies)]] == copies and np.all(got[:, len(copies):] == -1)

    def reserve(self, requests):
        slots, lens, new = zip(*requests)
        self.ora.empty = False
        copies = self.ora.reserve(requests)
        self.gpu.reserve([], len(requests), self.ints(slots), self.ints(lens), self.ints(np.concatenate([[0], np.cumsum(new)])))
        self.check(copies, len(requests))
        assert bool(self.gpu.status() & self.B.DEV_POOL_EMPTY) == self.ora.empty
        self.gpu.dev_status.zero_()
        return copies

    def fork(self, src, dst, lens):
        for a, b, n in zip(src, dst, lens):
            self.ora.fork(a, b, n)
        self.gpu.fork([], len(src), self.ints(src), self.ints(dst), self.ints(lens))
        self.check()

    def release(self, slots, keep=None):
        for k, s in enumerate(slots):
            self.ora.release(s, keep[k] if keep is not None else 0)
        self.gpu.release(len(slots), self.ints(slots), None if keep is None else self.ints(keep))
        self.check()

    def compact(self):
        moves, live = self.ora.compact()
        self.gpu.compact([])
        self.check(moves, (self.gpu.n_pages + 1) // 2)
        assert int(self.gpu.n_live.item()) == live


def test_shared_tails_are_copied_in_order():
    p = Pair(8, 6, 40)
    p.reserve([(0, 0, 200)])
    p.fork([0, 0, 0], [1, 2, 3], [200, 200, 200])
    assert len(p.reserve([(2, 200, 1), (0, 200, 100), (3, 200, 57)])) == 3       # slot 1 still holds the page
    assert p.reserve([(1, 200, 1)]) == []                                        # its only holder by now
    p.fork([1, 1], [4, 5], [200, 200])
    assert len(p.reserve([(5, 200, 1), (1, 200, 1), (4, 200, 1)])) == 2          # all holders at once: the last keeps it
    p.fork([1], [6], [192])                                                      # no partly filled page: nothing to copy
    assert p.reserve([(6, 192, 1), (0, 300, 1)]) == []
    p.release([0, 6, 0])                                                         # the same slot twice
    assert p.gpu.status() == 0


def test_an_empty_pool_hands_out_nothing_and_locks_shared_pages():
    p = Pair(4, 8, 7)
    p.reserve([(0, 0, 130)])
    p.fork([0], [1], [130])
    p.reserve([(2, 0, 192)])                                                     # six of seven pages are taken
    p.reserve([(0, 130, 1), (3, 0, 64)])                                         # two wanted, one free
    assert p.ora.table[0, 2] < -1 and p.ora.empty
    p.reserve([(3, 0, 64)])
    p.reserve([(1, 130, 1)])                                                     # the other holder is locked too
    p.fork([0], [3], [130])                                                      # a copy of a sequence with a locked entry (its page is given back first)
    p.compact()
    p.release([2])
    p.reserve([(0, 130, 1), (1, 130, 1), (3, 130, 1)])                           # now there is room: unlocked
    assert not p.ora.empty and p.ora.table.min() == -1


def test_a_locked_entry_whose_other_holders_are_gone_is_unlocked():
    p = Pair(3, 4, 2)
    p.reserve([(0, 0, 100)])
    p.fork([0], [1], [100])
    p.reserve([(0, 100, 1)])
    assert p.ora.empty and p.ora.table[0, 1] == -3
    p.release([1])
    assert p.reserve([(0, 100, 1)]) == [] and p.ora.table[0, 1] == 1


@pytest.mark.parametrize("n_slots,max_pages,n_pages", [(3, 1, 1), (5, 4, 9), (16, 40, 300), (40, 33, 5000), (700, 5, 4001), (9, 300, 40000)])
def test_random_calls_match_the_oracle(n_slots, max_pages, n_pages):
    rng = np.random.default_rng(n_pages)
    p, lens = Pair(n_slots, max_pages, n_pages), np.zeros(n_slots, int)
    for _ in range(14):
        op = rng.integers(0, 5)
        some = rng.permutation(n_slots)[:int(rng.integers(1, n_slots + 1))]
        if op <= 1:
            new = np.where(rng.random(len(some)) < 0.2, 0, rng.integers(1, 1 + 64 * max_pages // (2 if op else 30) + 1, len(some)))
            requests = [(int(s), int(lens[s]), int(n)) for s, n in zip(some, new)]
            p.reserve(requests)
            if not p.ora.empty:
                for s, length, n in requests:
                    if length + n <= 64 * max_pages:
                        lens[s] += n
        elif op == 2 and n_slots > 1:
            half = len(some) // 2
            pairs = [(s, d) for s, d in zip(some[:half], some[half:]) if np.all(p.ora.table[s, :-(-lens[s] // 64)] != -1)]
            if pairs:
                src, dst = zip(*pairs)
                p.fork(src, dst, lens[list(src)])
                lens[list(dst)] = lens[list(src)]
        elif op == 3:
            keep = rng.integers(0, lens[some] + 1)
            p.release(some, keep if rng.random() < 0.5 else None)
            lens[some] = [min(lens[s], 64 * int((p.ora.table[s] != -1).sum())) for s in some]
        else:
            p.compact()
        p.ora.check()


def test_many_sequences_that_share_few_pages():
    """More sequences than one tile of the ranking, all of them copies of five."""
    n = 1300
    p = Pair(n, 2, 3 * n, max_batch=n)
    p.reserve([(s, 0, 70) for s in range(5)])
    p.fork([s % 5 for s in range(5, n)], list(range(5, n)), [70] * (n - 5))
    order = np.random.default_rng(1).permutation(n)
    assert len(p.reserve([(int(s), 70, 3) for s in order])) == n - 5
    p.release(list(range(0, n, 2)))
    p.compact()
    assert p.gpu.status() == 0


def test_bad_slots_pages_and_counts_are_flagged():
    B = pytest.importorskip("paper_2609_38121_b200.binding")
    p = Pair(3, 4, 20)
    p.reserve([(0, 0, 100), (1, 0, 30)])
    before = p.gpu.page_table.clone(), p.gpu.refs.clone()
    same = lambda: p.torch.equal(before[0], p.gpu.page_table) and p.torch.equal(before[1], p.gpu.refs)  # noqa: E731

    def flagged(bit):
        st = p.gpu.status()
        p.gpu.dev_status.zero_()
        return st == bit
    p.gpu.fork([], 2, p.ints([0, -1]), p.ints([7, 2]), p.ints([100, 100]))
    assert flagged(B.DEV_BAD_SLOT) and same()
    p.gpu.release(2, p.ints([3, -5]))
    assert flagged(B.DEV_BAD_SLOT) and same()
    p.gpu.reserve([], 1, p.ints([4]), p.ints([0]), p.ints([0, 5]))
    assert flagged(B.DEV_BAD_SLOT) and same()
    p.gpu.reserve([], 1, p.ints([0]), p.ints([100]), p.ints([0, 200]))           # beyond the table
    assert flagged(B.DEV_PAGE_TABLE_FULL) and same()
    p.gpu.reserve([], 2, p.ints([0, 1]), p.ints([100, -3]), p.ints([0, 0, 4]))   # nothing new; a length that is none
    assert flagged(0) and same()
    p.gpu.fork([], 1, p.ints([1]), p.ints([2]), p.ints([100]))                   # more pages than the source has
    assert flagged(B.DEV_BAD_PAGE_ID) and p.gpu.page_table[2].tolist() == [int(before[0][1, 0]), -1, -1, -1]
    p.gpu.fork([], 1, p.ints([1]), p.ints([1]), p.ints([30]))                    # onto itself: as it was
    assert flagged(0) and p.torch.equal(p.gpu.page_table[1], before[0][1])
    p.gpu.release(1, p.ints([2]))
    assert flagged(0) and same()
    p.gpu.reserve([], 1, p.ints([2]), p.ints([40]), p.ints([0, 1]))              # a partly filled page that is not there: its tokens are lost
    assert flagged(B.DEV_BAD_PAGE_ID) and int(p.gpu.page_table[2, 0]) >= 0 and int(p.gpu.n_copies.item()) == 0
    p.gpu.release(1, p.ints([2]))
    assert flagged(0) and same()
    p.gpu.page_table[2, 0] = 20                                                  # no page of the pool
    p.gpu.release(1, p.ints([2]))
    assert flagged(B.DEV_BAD_PAGE_ID) and same()
    p.gpu.page_table[2, 0] = 19                                                  # a free page that an entry names
    p.gpu.release(1, p.ints([2]))
    assert flagged(B.DEV_BAD_REFS) and same()
    p.gpu.page_table[2, 0] = 19
    p.gpu.compact([])
    assert flagged(B.DEV_BAD_REFS) and same()
    with pytest.raises(ValueError):
        p.gpu.reserve([], 4, p.ints([0] * 4), p.ints([0] * 4), p.ints([0] * 5))


@pytest.mark.parametrize("bits", [2, 3, 4])
def test_copies_of_pages_and_windows(bits):
    import torch
    from paper_2609_38121_b200 import binding as B
    n_kv, n_pages, cap = 3, 37, 70
    T = np.broadcast_to(np.eye(128, dtype=np.float32), (n_kv, 128, 128))
    pool = B.PagePool(6, 640, n_pages)
    c = B.PagedCache(6, n_kv, bits, 6, 640, 4, 64, 1, 0.96, 0.92, T, T, ring_cap=cap, pool=pool, page_bounds=True)
    gen = torch.Generator(device="cuda").manual_seed(bits)
    for t in (c.pages, c.bounds, c.exponents):
        t.copy_(torch.randint(0, 127, t.shape, generator=gen, device="cuda").to(t.dtype))
    for t in (c.ring_kv, c.sink_kv):
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    want = [t.clone() for t in (c.pages.view(n_pages, -1), c.bounds, c.exponents)]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    src, dst = [3, 36, 0, -1, 5], [4, 1, 35, -1, 5]
    for a, b in ((3, 4), (36, 1)):
        for t in want:
            t[b] = t[a]
    B.copy_pages(c.desc, 5, ints(src), ints(dst), ints([2]), c.bounds, c.exponents)                 # two of the list
    for t, w in zip((c.pages.view(n_pages, -1), c.bounds, c.exponents), want):
        assert torch.equal(t, w)
    want[0][35] = want[0][0]
    B.copy_pages(c.desc, 5, ints(src), ints(dst), ints([9]))                                        # a count beyond the capacity; no bounds
    for t, w in zip((c.pages.view(n_pages, -1), c.bounds, c.exponents), want):
        assert torch.equal(t, w)
    assert c.status() == 0
    B.copy_pages(c.desc, 2, ints([37, 2]), ints([2, -4]), ints([2]))
    assert c.status() == B.DEV_BAD_PAGE_ID and torch.equal(c.pages.view(n_pages, -1), want[0])
    c.dev_status.zero_()
    ring, sink = c.ring_kv.clone(), c.sink_kv.clone()
    for a, b, n in ((0, 3, 2), (1, 4, 69), (2, 5, 500)):
        ring[b, :, :, :min(n, cap)], sink[b, :, :, :min(n, 4)] = ring[a, :, :, :min(n, cap)], sink[a, :, :, :min(n, 4)]
    B.copy_windows(c.desc, 4, ints([0, 1, 2, 1]), ints([3, 4, 5, 1]), ints([2, 69, 500, 30]))
    assert torch.equal(ring, c.ring_kv) and torch.equal(sink, c.sink_kv) and c.status() == 0
    B.copy_windows(c.desc, 2, ints([0, 6]), ints([-1, 1]), ints([9, 9]))
    assert torch.equal(ring, c.ring_kv) and c.status() == B.DEV_BAD_SLOT
    B.copy_windows(c.desc, 1, ints([0]), ints([1]), ints([0]))                                      # an empty source
    assert torch.equal(ring, c.ring_kv) and torch.equal(sink, c.sink_kv)


class Server:
    """Sequences in a pool (two layers that share one page table) beside reference caches with pages of their own."""

    def __init__(self, n_slots, max_len, n_pages, bits=2, n_q=8, n_kv=2, seed=5):
        import torch
        from paper_2609_38121_b200 import binding as B
        self.torch, self.B, self.max_len, self.n_slots, self.n_q, self.n_kv = torch, B, max_len, n_slots, n_q, n_kv
        self.wl = W.LayerWorkload(dict(seed=seed, batch=1, n_q=n_q, n_kv=n_kv, ctx=0, theta=1e4, bits=bits, s_sink=4, s_keep=64, rmsnorm=False, ragged=None,
                                       prefill_chunk=0))
        T, Ti, _ = oracle_transforms(self.wl)
        self.pool = B.PagePool(n_slots, max_len, n_pages)
        make = lambda **kw: B.PagedCache(n_q, n_kv, bits, n_slots, max_len, 4, 64, 1, 0.96, 0.92, T, Ti, page_bounds=True, **kw)  # noqa: E731
        self.layers, self.own = [make(pool=self.pool) for _ in range(2)], [make() for _ in range(2)]
        self.tokens = {}                                       # slot: list of (layer 0 K, V, layer 1 K, V) rows

    def ints(self, v):
        return self.torch.tensor([int(x) for x in v], dtype=self.torch.int32, device="cuda")

    def append(self, slots, counts, rng, reserve=True):
        """New random tokens for the slots: in the pool as they are, in the reference caches the same ones."""
        torch, B = self.torch, self.B
        lens, cu = [len(self.tokens.get(s, [])) for s in slots], self.ints(np.concatenate([[0], np.cumsum(counts)]))
        if reserve:
            self.pool.reserve(self.layers, len(slots), self.ints(slots), self.ints(lens), cu)
        rows = [[W.f32_to_bf16_bits(rng.standard_normal((4, self.n_kv, 128)).astype(np.float32) * 2).view(np.int16) for _ in range(c)] for c in counts]
        flat = np.stack([r for group in rows for r in group])
        for i in range(2):
            K, V = (torch.from_numpy(np.ascontiguousarray(flat[:, 2 * i + k])).cuda() for k in range(2))
            for cache in (self.layers[i], self.own[i]):
                seq_len = self.ints(lens)
                B.append(cache.desc, len(slots), self.ints(slots), seq_len, cu, sum(counts), max(counts), K, V)
                B.update_page_bounds(cache.desc, len(slots), self.ints(slots), seq_len, cu, max(counts), cache.bounds, cache.exponents)
                assert seq_len.tolist() == [n + c for n, c in zip(lens, counts)]
        for s, group in zip(slots, rows):
            self.tokens.setdefault(s, []).extend(group)

    def fork(self, src, dst, rng):
        lens = [len(self.tokens[s]) for s in src]
        self.pool.fork(self.layers, len(src), self.ints(src), self.ints(dst), self.ints(lens))
        for a, b in zip(src, dst):
            self.tokens[b] = list(self.tokens[a])
            for cache in self.own:                             # the reference: pages of its own, everything copied
                pa, pb = cache.page_table[a].long(), cache.page_table[b].long()
                for t in (cache.pages.view(-1, cache.page_bytes), cache.bounds, cache.exponents):
                    t[pb] = t[pa]
                cache.ring_kv[b], cache.sink_kv[b] = cache.ring_kv[a], cache.sink_kv[a]

    def release(self, slots):
        self.pool.release(len(slots), self.ints(slots))
        for s in slots:
            del self.tokens[s]

    def check(self, rng, n_select=3):
        """Dense and sparse attention of all sequences: the same bits from the pool as from the reference caches."""
        torch, B = self.torch, self.B
        slots = sorted(self.tokens)
        lens = self.ints([len(self.tokens[s]) for s in slots])
        Q = torch.from_numpy(W.f32_to_bf16_bits(rng.standard_normal((len(slots), self.n_q, 128)).astype(np.float32)).view(np.int16)).cuda()
        n = len(slots)
        for a, b in zip(self.layers, self.own):
            got = []
            for c in (a, b):
                O, O16 = torch.empty((n, self.n_q, 128), device="cuda"), torch.empty((n, self.n_q, 128), dtype=torch.bfloat16, device="cuda")
                sel = torch.empty((n, self.n_kv, n_select), dtype=torch.int32, device="cuda")
                need = max(B.decode_workspace_bytes(c.desc, n, self.max_len), B.sparse_workspace_bytes(c.desc, n, self.max_len, n_select))
                ws = torch.empty(need, dtype=torch.uint8, device="cuda")
                B.decode_attn(c.desc, n, self.ints(slots), lens, self.max_len, Q, O, ws, need)
                B.decode_attn_sparse(c.desc, n, self.ints(slots), lens, self.max_len, Q, c.bounds, c.exponents, n_select, sel, O16, ws, need)
                got.append((O, sel, O16))
                assert c.status() == 0
            for x, y in zip(*got):
                assert torch.equal(x, y) and torch.all(torch.isfinite(x.float()))
        assert self.pool.status() == 0
        refs, table = self.pool.refs.cpu().numpy(), self.pool.page_table.cpu().numpy()
        named = np.zeros_like(refs)
        np.add.at(named, table[table >= 0], 1)
        assert np.array_equal(named, refs)


@pytest.mark.parametrize("bits", [2, 3, 4])
def test_beams_prefixes_and_compaction_leave_every_sequence_as_its_own(bits):
    rng = np.random.default_rng(bits)
    s = Server(8, 640, 48, bits=bits)
    s.append([0, 1], [300, 131], rng)
    s.fork([0, 0, 1], [2, 3, 4], rng)
    s.check(rng)
    s.append([0, 2, 3, 4], [1, 1, 1, 1], rng)                  # the copies go separate ways
    s.append([3, 1, 2], [70, 200, 1], rng)
    s.check(rng)
    s.release([0, 4])
    s.pool.compact(s.layers)
    assert int(s.pool.n_live.item()) == int((s.pool.refs > 0).sum()) and int((s.pool.refs[int(s.pool.n_live.item()):] > 0).sum()) == 0
    s.check(rng)
    s.fork([2], [3], rng)                                       # onto a slot that held another sequence
    s.append([5, 3, 2], [250, 3, 1], rng)
    s.check(rng)
    s.pool.compact(s.layers)
    s.append([1, 2, 3, 5], [1, 1, 1, 1], rng)
    s.check(rng)


def test_a_locked_sequence_cannot_write_into_a_shared_page():
    rng = np.random.default_rng(77)
    s = Server(4, 256, 4)
    s.append([0], [100], rng)
    s.fork([0], [1], rng)
    s.append([2], [128], rng)                                   # the pool is full
    want = s.layers[0].pages.clone()
    one = s.torch.zeros((1, 2, 128), dtype=s.torch.int16, device="cuda")
    s.pool.reserve(s.layers, 1, s.ints([1]), s.ints([100]), s.ints([0, 1]))
    assert s.pool.status() == s.B.DEV_POOL_EMPTY
    seq_len = s.ints([100])
    s.B.append(s.layers[0].desc, 1, s.ints([1]), seq_len, s.ints([0, 1]), 1, 1, one, one)
    assert s.layers[0].status() == s.B.DEV_BAD_PAGE_ID and seq_len.tolist() == [100] and s.torch.equal(want, s.layers[0].pages)
    s.pool.dev_status.zero_()
    s.layers[0].dev_status.zero_()
    s.release([2])
    s.append([1], [1], rng)
    s.check(rng)


def test_reserve_fork_and_copies_in_a_captured_graph():
    """A beam step (fork, reserve, copies) captured once and replayed: each replay gives the state of the plain calls."""
    import torch
    from paper_2609_38121_b200 import binding as B
    states = []
    for captured in (False, True):
        rng = np.random.default_rng(4)
        s = Server(4, 320, 30)
        s.append([0, 1], [100, 200], rng)
        src, dst, lens, cu = s.ints([0, 1]), s.ints([2, 3]), s.ints([100, 200]), s.ints([0, 1, 2])

        def step(stream=None):
            s.pool.fork(s.layers, 2, src, dst, lens, stream)
            s.pool.reserve(s.layers, 2, dst, lens, cu, stream)

        if captured:
            stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                step(stream)
        for i in range(3):
            graph.replay() if captured else step()
            src.copy_(s.ints([1, 0]))
            lens.copy_(s.ints([200, 100]))
            torch.cuda.synchronize()
        states.append([t.clone() for t in (s.pool.page_table, s.pool.refs, s.layers[0].pages, s.layers[1].ring_kv, s.layers[1].bounds)])
        assert s.pool.status() == 0
    for a, b in zip(*states):
        assert torch.equal(a, b)
