"""Appends that cannot store all tokens of a sequence store none of them: its length, windows and pages stay as they were, dense and
sparse attention at that length give the same bits as before, and the other sequences of the call get what they get without it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

MISSING, LOCKED, BEYOND, LOWEST = -1, -2, 1 << 20, -(1 << 31)


class Twins:
    """Two caches with the same contents; entries of the first one's page table are damaged before the call under test."""

    def __init__(self, have, n_kv=2, G=2, bits=2, max_pages=8, kappa=0.96, quantizer=0, s_sink=4, prologue=False, seed=1):
        import torch
        from paper_2609_38121_b200 import binding as B
        self.torch, self.B, self.n_kv, self.G, self.n = torch, B, n_kv, G, len(have)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        T = np.stack([np.linalg.qr(rng.standard_normal((128, 128)))[0] for _ in range(n_kv)]).astype(np.float32)
        self.max_len, self.max_pages = 64 * max_pages, max_pages
        order = rng.permutation(self.n * max_pages)
        self.caches = [B.PagedCache(n_kv * G, n_kv, bits, self.n, self.max_len, s_sink, 64, 1, kappa, kappa, T, T, quantizer=quantizer, page_order=order,
                                    page_bounds=True) for _ in range(2)]
        self.prologue = B.Prologue(1e4, self.max_len + 64) if prologue else None
        self.slot = self.ints(range(self.n))
        self.lens = [self.ints([0] * self.n) for _ in range(2)]
        self.append(have)
        assert all(c.status() == 0 for c in self.caches) and self.lens[0].tolist() == list(have)

    def ints(self, v):
        return self.torch.tensor([int(x) for x in v], dtype=self.torch.int32, device="cuda")

    def append(self, counts, slots=None):
        torch, B, total = self.torch, self.B, int(sum(counts))
        cu = self.ints(np.concatenate([[0], np.cumsum(counts)]))
        K, V = (torch.randn((total, self.n_kv, 128), generator=self.gen, device="cuda").to(torch.bfloat16).view(torch.int16) for _ in range(2))
        for i, c in enumerate(self.caches):
            slot = self.slot if slots is None or i else self.ints(slots)
            if self.prologue is None:
                B.append(c.desc, self.n, slot, self.lens[i], cu, total, max(counts), K, V)
            else:
                B.append_projected(c.desc, self.n, slot, self.lens[i], cu, total, max(counts), K, V, self.prologue.desc)
            B.update_page_bounds(c.desc, self.n, self.slot, self.lens[i], cu, max(counts), c.bounds, c.exponents)

    def state(self, i):
        c = self.caches[i]
        return [t.clone() for t in (c.pages.view(-1, c.page_bytes), c.ring_kv, c.sink_kv)]

    def attend(self, i, rows):
        """Dense and sparse attention of some of the sequences, a call each (the split over the GPU then is the same every time)."""
        torch, B, c = self.torch, self.B, self.caches[i]
        Q = torch.randn((1, self.n_kv * self.G, 128), generator=torch.Generator(device="cuda").manual_seed(9), device="cuda").to(torch.bfloat16).view(torch.int16)
        need = max(B.decode_workspace_bytes(c.desc, 1, self.max_len), B.sparse_workspace_bytes(c.desc, 1, self.max_len, 2))
        ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), []
        for b in rows:
            O, O16 = torch.empty((1, self.n_kv * self.G, 128), device="cuda"), torch.empty((1, self.n_kv * self.G, 128), dtype=torch.bfloat16, device="cuda")
            sel = torch.empty((1, self.n_kv, 2), dtype=torch.int32, device="cuda")
            B.decode_attn(c.desc, 1, self.slot[b:b + 1], self.lens[i][b:b + 1], self.max_len, Q, O, ws, need)
            B.decode_attn_sparse(c.desc, 1, self.slot[b:b + 1], self.lens[i][b:b + 1], self.max_len, Q, c.bounds, c.exponents, 2, sel, O16, ws, need)
            out += [O, sel, O16]
        return out

    def check(self, counts, damage, bits, slots=None):
        """damage: sequence -> {table index: entry} (of its first new page or behind it)."""
        torch, B = self.torch, self.B
        refused = set(damage) | {b for b, s in enumerate(slots or []) if not 0 <= s < self.n}
        have, (a, twin) = self.lens[0].tolist(), self.caches
        rows = [b for b in refused if 0 < have[b] <= self.max_len]
        before, attended = self.state(0), self.attend(0, rows)
        saved = a.page_table.clone()
        for b, entries in damage.items():
            for i, e in entries.items():
                if i < self.max_pages:
                    a.page_table[b, i] = -2 - int(saved[b, i]) if e == LOCKED else e
        self.append(counts, slots)
        status = a.status()
        a.page_table.copy_(saved)
        got, other = self.state(0), self.state(1)
        want = [t.clone() for t in before]
        for b in set(range(self.n)) - refused:
            pages = saved[b].long()
            want[0][pages] = other[0][pages]
            want[1][b], want[2][b] = other[1][b], other[2][b]
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        assert status & (B.DEV_PAGE_TABLE_FULL | B.DEV_BAD_PAGE_ID | B.DEV_BAD_SLOT) == bits
        assert self.lens[0].tolist() == [n if b in refused else n + c for b, (n, c) in enumerate(zip(have, counts))]
        for x, y in zip(attended, self.attend(0, rows)):
            assert torch.equal(x, y)
        a.dev_status.zero_()                                    # the twin goes on from the same state
        for x, y in ((a.pages, twin.pages), (a.ring_kv, twin.ring_kv), (a.sink_kv, twin.sink_kv), (a.bounds, twin.bounds), (a.exponents, twin.exponents),
                     (self.lens[0], self.lens[1])):
            y.copy_(x)


@pytest.mark.parametrize("bits,entry", [(2, MISSING), (3, LOCKED), (4, BEYOND), (2, LOWEST)])
def test_a_few_tokens_across_a_page_boundary(bits, entry):
    """A warp per token: positions 120 .. 127 have a page, 128 .. 129 have none; their ring rows hold positions 56 .. 63."""
    t = Twins([120, 126, 60, 0, 127], bits=bits)
    t.check([10, 4, 10, 3, 2], {0: {2: entry}, 4: {2: entry}}, t.B.DEV_BAD_PAGE_ID)
    t.check([10, 4, 70, 70, 2], {0: {1: entry}, 2: {1: entry}, 3: {0: entry}}, t.B.DEV_BAD_PAGE_ID)


@pytest.mark.parametrize("prologue", [False, True])
def test_many_short_chunks(prologue):
    """The tensor-core path for short chunks: a warp of tokens holds several sequences, whole ones and parts of longer ones."""
    rng = np.random.default_rng(4)
    n = 60
    have, new = rng.integers(40, 130, n), rng.integers(1, 100, n)
    new[20:30] = rng.integers(1, 6, 10)
    have[22], new[22], new[9] = 126, 4, 0
    t = Twins(have, n_kv=8, G=1, bits=3, prologue=prologue)
    damage = {b: {(have[b] + new[b] - 1) // 64: MISSING} for b in range(n) if new[b] and b % 3 == 1}
    damage[40] = {int(have[40]) // 64: LOCKED}
    assert 22 in damage and sum(new) > 2000
    t.check(new, damage, t.B.DEV_BAD_PAGE_ID)


@pytest.mark.parametrize("bits,kappa,quantizer", [(2, 0.96, 0), (4, 0.9, 0), (3, 0.7, 0), (4, 0.96, 1)])
def test_chunks(bits, kappa, quantizer):
    """Long chunks, with every quantizer: the missing page is the first, the last and one in the middle; single tokens between them."""
    t = Twins([100, 0, 64, 200, 1, 130], bits=bits, kappa=kappa, quantizer=quantizer, max_pages=12)
    t.check([300, 400, 1, 129, 500, 1], {0: {1: MISSING}, 3: {5: LOCKED}, 4: {4: BEYOND}}, t.B.DEV_BAD_PAGE_ID)
    t.check([1, 200, 300, 2, 131, 64], {1: {7: MISSING}, 4: {2: MISSING}, 5: {3: MISSING}}, t.B.DEV_BAD_PAGE_ID)


def test_a_page_far_behind():
    """More pages than a warp looks at in one round, checked once for many tiles."""
    t = Twins([70, 10, 129], n_kv=1, max_pages=720)
    t.check([45000, 200, 45000], {0: {699: MISSING}}, t.B.DEV_BAD_PAGE_ID)
    t.check([45000, 200, 7], {2: {705: MISSING}}, t.B.DEV_BAD_PAGE_ID)


@pytest.mark.parametrize("longest", [20, 150])
def test_beyond_the_table_and_bad_slots(longest):
    t = Twins([100, 470, 30])
    t.check([20, 5, longest], {}, 0)
    t.check([longest, 6, 10], {}, t.B.DEV_BAD_SLOT, slots=[0, 1, -3])
    t.check([7, 6, longest], {}, t.B.DEV_BAD_SLOT, slots=[0, 3, 2])
    t.check([longest, 32, 60], {1: {8: MISSING}}, t.B.DEV_PAGE_TABLE_FULL)       # the table ends at 512 positions: 481 + 32
    past = {2: {8: MISSING}} if longest == 150 else {}                            # 30 + 150 + 10 + 150 + 60 + 150 tokens, or 30 + 20 + 10 + 20 + 60 + 20
    t.check([1, 31, longest], past, t.B.DEV_PAGE_TABLE_FULL if past else 0)


def test_lengths_at_the_end_of_32_bits():
    """Positions that 32 bits do not hold are behind the table's end."""
    t = Twins([100, 90])
    before = t.state(0)
    t.lens[0].copy_(t.ints([2 ** 31 - 3, 2 ** 31 - 70]))
    t.lens[1].copy_(t.ints([2 ** 31 - 3, 2 ** 31 - 70]))
    for counts in ([3, 60], [200, 140]):
        t.append(counts)
        assert t.caches[0].status() == t.B.DEV_PAGE_TABLE_FULL and t.lens[0].tolist() == [2 ** 31 - 3, 2 ** 31 - 70]
        for x, y in zip(t.state(0), before):
            assert t.torch.equal(x, y)


@pytest.mark.parametrize("n_new", [3, 130])
def test_rows_behind_the_last_sequence_are_left_alone(n_new):
    """Keys and values of a padded call: more rows than the sequences bring."""
    torch = pytest.importorskip("torch")
    t = Twins([100, 90])
    cu = t.ints([0, n_new, n_new + 2])
    K, V = (torch.randn((n_new + 9, 2, 128), generator=t.gen, device="cuda").to(torch.bfloat16).view(torch.int16) for _ in range(2))
    for i, rows in enumerate((n_new + 9, n_new + 2)):
        t.B.append(t.caches[i].desc, 2, t.slot, t.lens[i], cu, rows, n_new, K, V)
    for x, y in zip(t.state(0), t.state(1)):
        assert torch.equal(x, y)
    assert t.lens[0].tolist() == [100 + n_new, 92] and t.caches[0].status() == 0
