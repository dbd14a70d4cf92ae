"""Random sessions of a server: appends of any size, forks, lengths that go back with and without a release, compaction, in pools that
run empty.  After every call all sequences attend, densely and sparsely, with the same bits as in caches that share nothing, and table
and counts are the oracle's."""
import numpy as np
import pytest

from oracle import sparse_oracle as S
from paper_2609_38121_b200 import workloads as W
from tests.test_gpu_page_pool import Server

pytestmark = pytest.mark.gpu


class Session(Server):
    def __init__(self, seed, bits, n_slots, max_pages, n_pages, n_kv):
        super().__init__(n_slots, 64 * max_pages, n_pages, bits=bits, n_q=4 * n_kv, n_kv=n_kv, seed=seed)
        self.rng, self.ora, self.lens = np.random.default_rng(seed), S.Pool(n_slots, max_pages, n_pages), [0] * n_slots
        self.refused = 0

    def some(self):
        return [int(x) for x in self.rng.permutation(self.n_slots)[:int(self.rng.integers(1, self.n_slots + 1))]]

    def step(self):
        """Reserve, append and bounds for some of the sequences; those that are refused stay as they are."""
        torch, B, rng = self.torch, self.B, self.rng
        slots = self.some()
        counts = [int(rng.integers(len(slots) == 1, [2, 6, 90, 260][int(rng.integers(0, 4))])) for _ in slots]
        lens, n = [self.lens[k] for k in slots], len(slots)
        cu, ids, total, most = self.ints(np.concatenate([[0], np.cumsum(counts)])), self.ints(slots), sum(counts), max(counts)
        if total == 0:
            return
        self.pool.reserve(self.layers, n, ids, self.ints(lens), cu)
        self.ora.empty = False
        self.ora.reserve(list(zip(slots, lens, counts)))
        assert bool(self.pool.status() & B.DEV_POOL_EMPTY) == self.ora.empty
        self.pool.dev_status.zero_()
        for layer, own in zip(self.layers, self.own):
            K, V = (torch.from_numpy(W.f32_to_bf16_bits(rng.standard_normal((total, self.n_kv, 128)).astype(np.float32) * 2).view(np.int16)).cuda() for _ in range(2))
            after = self.ints(lens)
            B.append(layer.desc, n, ids, after, cu, total, most, K, V)
            stored = [a == x + c for a, x, c in zip(after.tolist(), lens, counts)]
            assert all(ok or a == x for ok, a, x in zip(stored, after.tolist(), lens)) and (all(stored) or layer.status() != 0)
            layer.dev_status.zero_()
            # the reference takes the same call (the same path through the library) and puts back what the pool's refused
            pages = own.pages.view(-1, own.page_bytes)
            back = [(k, own.ring_kv[k].clone(), own.sink_kv[k].clone(), pages[own.page_table[k].long()]) for k, ok in zip(slots, stored) if not ok]
            own_after = self.ints(lens)
            B.append(own.desc, n, ids, own_after, cu, total, most, K, V)
            own.dev_status.zero_()
            for k, ring, sink, rows in back:
                own.ring_kv[k], own.sink_kv[k] = ring, sink
                pages[own.page_table[k].long()] = rows
            cu_stored = self.ints(np.concatenate([[0], np.cumsum([c * ok for c, ok in zip(counts, stored)])]))
            for cache in (layer, own):
                B.update_page_bounds(cache.desc, n, ids, after, cu_stored, most, cache.bounds, cache.exponents)
        self.refused += len(back)
        for k, a in zip(slots, after.tolist()):
            self.lens[k] = a

    def beams(self):
        order, half = [int(x) for x in self.rng.permutation(self.n_slots)], self.n_slots // 2
        pairs = [(a, b) for a, b in zip(order[:half], order[half:]) if self.lens[a]]
        if not pairs:
            return
        src, dst = zip(*pairs)
        lens = [self.lens[a] for a in src]
        self.pool.fork(self.layers, len(src), self.ints(src), self.ints(dst), self.ints(lens))
        for a, b, n in zip(src, dst, lens):
            self.ora.fork(a, b, n)
            self.lens[b] = n
            for cache in self.own:
                pa, pb = cache.page_table[a].long(), cache.page_table[b].long()
                for t in (cache.pages.view(-1, cache.page_bytes), cache.bounds, cache.exponents):
                    t[pb] = t[pa]
                for t in (cache.ring_kv, cache.sink_kv):
                    rows = min(n, t.shape[3])
                    t[b][:, :, :rows] = t[a][:, :, :rows]

    def go_back(self):
        for k in self.some():
            self.lens[k] = [self.lens[k] // 64 * 64, int(self.rng.integers(0, self.lens[k] + 1))][int(self.rng.integers(0, 2))]

    def give_back(self):
        slots = self.some()
        keep = [int(self.rng.integers(0, self.lens[k] + 1)) * int(self.rng.integers(0, 2)) for k in slots]
        self.pool.release(len(slots), self.ints(slots), self.ints(keep))
        for k, n in zip(slots, keep):
            self.ora.release(k, n)
            self.lens[k] = n

    def pack(self):
        self.pool.compact(self.layers)
        self.ora.compact()

    def compare(self):
        torch, B = self.torch, self.B
        slots = [k for k, n in enumerate(self.lens) if n]
        n, lens, ids = len(slots), self.ints([self.lens[k] for k in slots]), self.ints(slots)
        Q = torch.from_numpy(W.f32_to_bf16_bits(self.rng.standard_normal((max(n, 1), self.n_q, 128)).astype(np.float32)).view(np.int16)).cuda()
        for pair in zip(self.layers, self.own) if n else ():
            got = []
            for c in pair:
                O, O16 = torch.empty((n, self.n_q, 128), device="cuda"), torch.empty((n, self.n_q, 128), dtype=torch.bfloat16, device="cuda")
                sel = torch.empty((n, self.n_kv, 3), dtype=torch.int32, device="cuda")
                need = B.decode_workspace_bytes(c.desc, n, self.max_len)
                B.decode_attn(c.desc, n, ids, lens, self.max_len, Q, O, torch.empty(need, dtype=torch.uint8, device="cuda"), need)
                B.decode_attn_sparse(c.desc, n, ids, lens, self.max_len, Q, c.bounds, c.exponents, 3, sel, O16)
                assert c.status() == 0
                got.append((O, sel, O16))
            for x, y in zip(*got):
                assert torch.equal(x, y) and bool(torch.isfinite(x.float()).all())
        assert self.pool.status() == 0
        assert np.array_equal(self.pool.page_table.cpu().numpy(), self.ora.table) and np.array_equal(self.pool.refs.cpu().numpy(), self.ora.refs)
        self.ora.check()


@pytest.mark.parametrize("seed,bits,n_slots,max_pages,n_pages,n_kv", [(1, 2, 5, 8, 20, 2), (2, 3, 8, 5, 17, 1), (3, 4, 3, 12, 20, 2), (4, 2, 7, 3, 9, 8), (5, 3, 4, 9, 40, 8),
                                                                      (6, 4, 8, 6, 26, 1)])
def test_sessions(seed, bits, n_slots, max_pages, n_pages, n_kv):
    s = Session(seed, bits, n_slots, max_pages, n_pages, n_kv)
    calls = [s.step] * 4 + [s.beams, s.go_back, s.give_back, s.pack]
    for _ in range(50):
        calls[int(s.rng.integers(0, len(calls)))]()
        s.compare()
    assert s.refused > 0
