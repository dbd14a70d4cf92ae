"""Sparse decode attention on the GPU against the oracle: page bounds and selected pages are equal number by number, outputs
within the decode tolerance plus the rounding to bf16."""
import numpy as np
import pytest

from oracle import sparse_oracle as S
from oracle import wushkv_oracle as O
from paper_2609_38121_b200 import workloads as W
from tests.harness import DECODE_TOL, Layer

pytestmark = pytest.mark.gpu

SCALE = 1.0 / np.sqrt(128)
BF16_HALF_STEP = 2.0 ** -8          # rounding of the output, relative to it


def _wl(n_q, n_kv, seed, batch, bits=2, s_keep=64, rmsnorm=False):
    return W.LayerWorkload(dict(seed=seed, batch=batch, n_q=n_q, n_kv=n_kv, ctx=0, theta=1e4, bits=bits, s_sink=4,
                                s_keep=s_keep, rmsnorm=rmsnorm, ragged=None, prefill_chunk=0))


class Sparse:
    """A filled layer with bounds of its pages."""

    def __init__(self, lengths, n_q=8, n_kv=2, bits=2, s_sink=4, s_keep=64, s_flush=1, seed=71, lag=0, quantizer="affine", fill=True, rmsnorm=False, **kw):
        import torch
        from paper_2609_38121_b200 import binding as B
        self.torch, self.B = torch, B
        self.wl = _wl(n_q, n_kv, seed, len(lengths), bits, s_keep, rmsnorm)
        self.L = Layer(self.wl, lengths, bits, s_sink, s_keep, s_flush, lag=lag, page_shuffle_seed=seed, quantizer=quantizer, **kw)
        n = self.L.cache.desc.n_pages
        self.bounds = torch.full((n, n_kv, 2, 128), 77, dtype=torch.int8, device="cuda")
        self.exponents = torch.full((n, n_kv), 99, dtype=torch.int8, device="cuda")
        # what was in the pool before: steps and offsets that are not numbers
        self.L.cache.pages.fill_(0xFF)
        self.pages_of = {}
        if fill:
            self.append(self.L.lengths)

    def append(self, counts):
        self.L.append_step(counts, oracle_too=False)
        self.L.lengths = list(self.L.done)            # the windows that are read back are those of the present lengths
        self.update(counts)

    def update(self, counts, max_new=None):
        cu = self.torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), device="cuda")
        self.B.update_page_bounds(self.L.cache.desc, self.L.batch, self.L.slot, self.L.seq_len, cu, max(counts) if max_new is None else max_new,
                                  self.bounds, self.exponents)

    def oracle_bounds(self, b, h):
        """(lower, upper, e) of all pages of a sequence and head, from the codes the GPU stored."""
        n = self.L.done[b]
        codes, step, zero = self.L.gpu_codes(b, h, 0, n=n)
        meta = np.stack([step, zero], axis=1)
        parts = [S.page_bounds(codes[i:i + 64].astype(np.int64), meta[i:i + 64]) for i in range(0, n, 64)]
        return tuple(np.stack([np.asarray(p[k]) for p in parts]) for k in range(3))

    def check_bounds(self):
        bounds, e = self.bounds.cpu().numpy().astype(int), self.exponents.cpu().numpy().astype(int)
        table, named = self.L.cache.page_table.cpu().numpy(), set()
        for b in range(self.L.batch):
            n = -(-self.L.done[b] // 64)
            pages = table[b, :n]
            named |= set(pages.tolist())
            for h in range(self.wl.n_kv):
                if n:
                    low, up, ex = self.oracle_bounds(b, h)
                    assert np.array_equal(bounds[pages, h, 0], low) and np.array_equal(bounds[pages, h, 1], up), (b, h)
                    assert np.array_equal(e[pages, h], ex), (b, h)
        others = np.array([p for p in range(len(bounds)) if p not in named], dtype=int)
        assert np.all(bounds[others] == 77) and np.all(e[others] == 99), "pages of nobody were written"

    def queries(self):
        q = np.stack([self.wl.queries(b, max(self.L.done[b] - 1, 0)) for b in range(self.L.batch)])
        return q, self.torch.from_numpy(W.f32_to_bf16_bits(q).view(np.int16)).cuda()

    def oracle_select(self, q, n_select):
        out = np.full((self.L.batch, self.wl.n_kv, n_select), -1, dtype=np.int64)
        G = self.wl.n_q // self.wl.n_kv
        for b in range(self.L.batch):
            _, _, first, n = S.packed_range(self.L.done[b], self.L.s_sink, self.L.s_keep, self.L.s_flush, self.L.lag)
            for h in range(self.wl.n_kv):
                if n:
                    low, up, e = (x[first:first + n] for x in self.oracle_bounds(b, h))
                    qc = [O.query_compensation(self.L.TinvT[h].astype(np.float32), q[b, h * G + g][None])[0] for g in range(G)]
                    out[b, h] = S.select(S.page_keys(qc, low, up, e, SCALE), n_select, first)
        return out

    def oracle_attention(self, b, q, pages, length=None):
        """pages [n_kv][...] of sequence b; queries [n_q][128]; length: of the row, if it is not the sequence's."""
        n, n_kv, G = length or self.L.done[b], self.wl.n_kv, self.wl.n_q // self.wl.n_kv
        kb, vb = self.L.gpu_window_arrays(b)
        out = np.zeros((self.wl.n_q, 128))
        for h in range(n_kv):
            kc, ks, kz = self.L.gpu_codes(b, h, 0, n=n)
            vc, vs, vz = self.L.gpu_codes(b, h, 1, n=n)
            K, V = O.effective_kv(kc, np.stack([ks, kz], 1), vc, np.stack([vs, vz], 1), kb[:n, h], vb[:n, h], n, self.L.s_sink, self.L.s_keep,
                                  self.L.s_flush, self.L.lag)
            lo, hi, _, _ = S.packed_range(n, self.L.s_sink, self.L.s_keep, self.L.s_flush, self.L.lag)
            for g in range(G):
                qc = O.query_compensation(self.L.TinvT[h], q[h * G + g][None])[0]
                out[h * G + g] = S.sparse_attention(qc, K, V, lo, hi, pages[h], SCALE)
        return out

    def sparse(self, Q, n_select, selected=None, max_seq_len=None, prologue=None, batch=None, slot=None, seq_len=None):
        """selected given: decode_attn_selected, else decode_attn_sparse.  Returns (selected, O) as arrays."""
        torch, B, c = self.torch, self.B, self.L.cache.desc
        batch = batch or self.L.batch
        slot, seq_len = self.L.slot if slot is None else slot, self.L.seq_len if seq_len is None else seq_len
        longest = max_seq_len or self.L.max_seq_len
        out = torch.full((batch, self.wl.n_q, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
        need = B.sparse_workspace_bytes(c, batch, longest, n_select)
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        if selected is None:
            sel = torch.full((batch, self.wl.n_kv, n_select), -9, dtype=torch.int32, device="cuda")
            B.decode_attn_sparse(c, batch, slot, seq_len, longest, Q, self.bounds, self.exponents, n_select, sel, out, ws, need, prologue=prologue)
            alone = torch.full_like(sel, -9)
            B.select_pages(c, batch, slot, seq_len, longest, Q, self.bounds, self.exponents, n_select, alone, prologue=prologue)
            assert torch.equal(sel, alone)
            again = torch.full_like(out, float("nan"))           # the list in the workspace
            B.decode_attn_sparse(c, batch, slot, seq_len, longest, Q, self.bounds, self.exponents, n_select, None, again, ws, need, prologue=prologue)
            assert torch.equal(out.view(torch.int16), again.view(torch.int16))
            again.fill_(float("nan"))                            # the list handed over
            B.decode_attn_selected(c, batch, slot, seq_len, longest, Q, sel, n_select, again, prologue=prologue)
            self.by_list = again.float().cpu().numpy().astype(np.float64)
        else:
            sel = torch.as_tensor(np.ascontiguousarray(selected, dtype=np.int32)).cuda()
            B.decode_attn_selected(c, batch, slot, seq_len, longest, Q, sel, n_select, out, prologue=prologue)
        torch.cuda.synchronize()
        return sel.cpu().numpy(), out.float().cpu().numpy().astype(np.float64)

    def check(self, n_select):
        q, Q = self.queries()
        sel, out = self.sparse(Q, n_select)
        assert np.array_equal(sel, self.oracle_select(q, n_select))
        for b in range(self.L.batch):
            if self.L.done[b] == 0:
                assert not out[b].any()
                continue
            _close(out[b], self.oracle_attention(b, q[b], sel[b]))
        assert self.L.cache.status() == 0
        return sel, out


def _close(out, ref):
    assert np.all(np.isfinite(out)) and np.all(np.isfinite(ref))
    slack = DECODE_TOL * np.abs(ref).max()
    worst = float(np.max(np.abs(out - ref) / (slack + BF16_HALF_STEP * (np.abs(ref) + slack))))
    assert worst <= 1.0


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (6, 2), (8, 2), (5, 1), (14, 2), (16, 2)])
def test_bounds_selection_and_attention_match_the_oracle(bits, n_q, n_kv):
    s = Sparse([1500, 0, 1, 68, 69, 333, 2050], n_q, n_kv, bits, seed=100 * bits + n_q)
    s.check_bounds()
    s.check(5)


@pytest.mark.parametrize("n_select", [1, 2, 31, 32, 33, 34, 200])
def test_every_number_of_pages(n_select):
    s = Sparse([2300, 700, 2116], seed=7)             # 35, 10 and 33 packed pages (32 behind 2116 - 64 positions and the sink's)
    s.check(n_select)


def test_all_pages_give_dense_attention():
    s = Sparse([1900, 640], 8, 2, 4, seed=8)
    q, Q = s.queries()
    _, out = s.sparse(Q, 64)
    dense, _ = s.L.decode(q)
    for b in range(2):
        _close(out[b], dense[b])


@pytest.mark.parametrize("s_sink,s_keep,s_flush,lag,quantizer", [(0, 64, 1, 0, "affine"), (4, 32, 16, 0, "quest"), (130, 64, 8, 0, "affine"), (4, 64, 1, 3, "affine")])
def test_windows_of_other_sizes(s_sink, s_keep, s_flush, lag, quantizer):
    s = Sparse([1111, 129, 211, 64 + s_sink], s_sink=s_sink, s_keep=s_keep, s_flush=s_flush, lag=lag, quantizer=quantizer, seed=9, n_q=6, n_kv=2)
    s.check_bounds()
    s.check(4)


def test_bounds_follow_the_appends():
    """Chunks, single tokens, sequences that bring nothing: always the bounds of exactly the tokens that are there."""
    s = Sparse([900, 900, 900], 4, 1, 3, seed=10, fill=False)
    for counts in ([70, 0, 1], [1, 1, 1], [57, 128, 62], [1, 0, 1], [300, 401, 1], [1, 1, 1]):
        s.append(counts)
        s.check_bounds()
    s.check(3)
    s.update([1, 1, 1], max_new=200)                  # a larger bound than any sequence brings
    s.check_bounds()


def test_more_pages_than_a_warp_step_and_many_sequences():
    s = Sparse([9000] + [150 + 37 * i for i in range(40)], 8, 2, 2, seed=11)
    s.check(17)


def test_more_heads_than_the_gpu_holds_at_once():
    """512 (sequence, KV head) pairs in several waves; some of them against the oracle, all of them finite; rows behind the batch stay."""
    lengths = [140 + (61 * i) % 500 for i in range(64)]
    s = Sparse(lengths, 32, 8, 4, seed=24)
    q, Q = s.queries()
    sel = s.torch.full((66, 8, 3), -9, dtype=s.torch.int32, device="cuda")
    out = s.torch.full((66, 32, 128), 7.0, dtype=s.torch.bfloat16, device="cuda")
    s.B.decode_attn_sparse(s.L.cache.desc, 64, s.L.slot, s.L.seq_len, s.L.max_seq_len, Q, s.bounds, s.exponents, 3, sel, out)
    sel, out = sel.cpu().numpy(), out.float().cpu().numpy().astype(np.float64)
    assert np.all(sel[64:] == -9) and np.all(out[64:] == 7.0) and np.all(np.isfinite(out))
    for b in (0, 17, 40, 63):
        first, n = S.packed_range(lengths[b], 4, 64, 1)[2:]
        for h in range(8):
            low, up, e = (x[first:first + n] for x in s.oracle_bounds(b, h))
            qc = [O.query_compensation(s.L.TinvT[h].astype(np.float32), q[b, h * 4 + g][None])[0] for g in range(4)]
            assert np.array_equal(sel[b, h], S.select(S.page_keys(qc, low, up, e, SCALE), 3, first))
        _close(out[b], s.oracle_attention(b, q[b], sel[b]))
    assert s.L.cache.status() == 0


def test_a_long_sequence_on_one_head_uses_a_cluster():
    s = Sparse([40000], 2, 1, 2, seed=12)
    s.check(40)


@pytest.mark.parametrize("n_q,n_kv", [(3, 1), (8, 1)])
def test_every_cluster_size_selects_the_same(n_q, n_kv):
    s = Sparse([40000, 9000, 3000], n_q, n_kv, 2, seed=22)
    q, Q = s.queries()
    ref = s.oracle_select(q, 624)
    for n_select in (1, 40, 150, 300, 624):
        want = ref if n_select == 624 else s.oracle_select(q, n_select)
        for cluster in (-1, 1, 2, 4, 8, 0):
            s.B.set_test_option("select_cluster", cluster)
            try:
                sel = s.torch.full((3, n_kv, n_select), -9, dtype=s.torch.int32, device="cuda")
                s.B.select_pages(s.L.cache.desc, 3, s.L.slot, s.L.seq_len, s.L.max_seq_len, Q, s.bounds, s.exponents, n_select, sel)
                assert np.array_equal(sel.cpu().numpy(), want), (n_select, cluster)
                # more pages with the same key than a bin's list holds
                s.B.select_pages(s.L.cache.desc, 3, s.L.slot, s.L.seq_len, s.L.max_seq_len, s.torch.zeros_like(Q), s.bounds, s.exponents, n_select, sel)
                pages = np.array([S.packed_range(n, 4, 64, 1)[3] for n in s.L.done])
                assert np.array_equal(sel.cpu().numpy()[:, 0], np.where(np.arange(n_select)[None] < np.minimum(pages, n_select)[:, None], np.arange(n_select)[None], -1))
            finally:
                s.B.set_test_option("select_cluster", 0)


def test_equal_keys_go_to_the_lower_page():
    s = Sparse([3000, 3000], 8, 2, 2, seed=13)
    s.bounds[:] = s.bounds[:1]
    s.exponents[:] = -5
    q, Q = s.queries()
    sel, out = s.sparse(Q, 6)
    assert np.array_equal(sel, np.broadcast_to(np.arange(6), sel.shape))
    for b in range(2):
        _close(out[b], s.oracle_attention(b, q[b], sel[b]))
    # a zero query and one that is not finite score 0 everywhere
    Q[0] = 0
    Q[1] = 0x7F80
    sel, out = s.sparse(Q, 6)
    assert np.array_equal(sel, np.broadcast_to(np.arange(6), sel.shape))
    _close(out[0], s.oracle_attention(0, np.zeros_like(q[0]), sel[0]))


@pytest.mark.parametrize("n_q,n_kv,bits", [(4, 1, 2), (8, 1, 4)])
def test_more_listed_pages_than_are_handed_over_in_shared_memory(n_q, n_kv, bits):
    s = Sparse([45000, 36000], n_q, n_kv, bits, seed=25)
    q, Q = s.queries()
    sel, out = s.sparse(Q, 560)
    assert np.array_equal(sel, s.oracle_select(q, 560))
    for b in range(2):
        _close(out[b], s.oracle_attention(b, q[b], sel[b]))


def test_lists_of_the_caller():
    """Any distinct pages in any order, places without a page anywhere, lists that leave the windows only."""
    s = Sparse([1500, 400, 1000], 6, 2, 4, seed=14)
    q, Q = s.queries()
    lists = np.full((3, 2, 7), -1)
    lists[0, 0], lists[0, 1] = [20, -1, 3, 0, 22, -1, 11], [5, 4, 3, 2, 1, 0, -1]
    lists[1, 0, :5], lists[1, 1, :5] = [5, 4, -1, 0, 1], [-1, -1, -1, -1, 2]     # six packed pages: six entries are read
    _, out = s.sparse(Q, 7, selected=lists)
    for b in range(3):
        _close(out[b], s.oracle_attention(b, q[b], lists[b]))
    assert s.L.cache.status() == 0
    # an index outside the packed pages is skipped and flagged; the others count
    lists[0, 0, 1], lists[0, 1, 6], lists[2, 0, 3] = 24, 1 << 30, -2
    _, out = s.sparse(Q, 7, selected=lists)
    lists[0, 0, 1], lists[0, 1, 6], lists[2, 0, 3] = -1, -1, -1
    for b in range(3):
        _close(out[b], s.oracle_attention(b, q[b], lists[b]))
    assert s.L.cache.status() == s.B.DEV_BAD_PAGE_ID


def test_several_rows_of_one_sequence():
    """Tokens to verify: the same slot with different lengths, each row as a sequence of that length."""
    s = Sparse([1300, 500], 8, 2, 2, seed=15, ring_cap=80)
    rows = [(0, 1300), (0, 1299), (0, 1290), (1, 500), (0, 1297), (1, 487)]
    ints = lambda k: s.torch.tensor([r[k] for r in rows], dtype=s.torch.int32, device="cuda")  # noqa: E731
    q = np.stack([s.wl.queries(b, n - 1) for b, n in rows])
    Q = s.torch.from_numpy(W.f32_to_bf16_bits(q).view(np.int16)).cuda()
    sel, out = s.sparse(Q, 4, batch=len(rows), slot=ints(0), seq_len=ints(1))
    for r, (b, n) in enumerate(rows):
        _close(out[r], s.oracle_attention(b, q[r], sel[r], length=n))
    assert s.L.cache.status() == 0


def test_projected_queries():
    """Norm and RoPE inside: the lists and outputs of the prepared queries, wherever their rounding to bf16 is beyond doubt."""
    from tests.test_gpu_projected import EPS, _prepared
    s = Sparse([1500, 800], 8, 2, 2, seed=16, rmsnorm=True)
    qp = np.stack([s.wl.projected(b, s.L.done[b])[1][-1] for b in range(2)])
    pro = s.B.Prologue(s.wl.theta, 2048, normalise=True, q_weight=s.wl.gain_q, eps=EPS)
    bits = lambda x: s.torch.from_numpy(W.f32_to_bf16_bits(x.astype(np.float32)).view(np.int16)).cuda()  # noqa: E731
    sel, out = s.sparse(bits(qp), 4, prologue=pro.desc)
    rounded = W.bf16_round_f32(qp.astype(np.float32))
    prepared, checked = [], 0
    for b in range(2):
        y, doubtful = _prepared(rounded[b][None], np.array([s.L.done[b] - 1]), s.wl.theta, s.wl.gain_q[None], True)
        prepared.append((y[0], doubtful[0]))
    plain_sel, plain_out = s.sparse(bits(np.stack([p[0] for p in prepared])), 4)
    for b in range(2):
        for h in range(2):
            if not prepared[b][1][4 * h:4 * h + 4].any():
                assert np.array_equal(sel[b, h], plain_sel[b, h]) and np.array_equal(out[b, 4 * h:4 * h + 4], plain_out[b, 4 * h:4 * h + 4])
                checked += 1
    assert checked >= 2 and s.L.cache.status() == 0
    short = s.B.Prologue(s.wl.theta, 1000, normalise=True, q_weight=s.wl.gain_q, eps=EPS)
    s.sparse(bits(qp), 4, prologue=short.desc)
    assert s.L.cache.status() == s.B.DEV_ROPE_RANGE


def test_bad_slots_tables_and_lengths_are_flagged():
    s = Sparse([1500, 1500, 1500], 8, 2, 2, seed=17)
    q, Q = s.queries()
    good_sel, good = s.sparse(Q, 4)
    slot = s.L.slot.clone()
    slot[1] = 3
    sel, out = s.sparse(Q, 4, slot=slot)
    assert s.L.cache.status() == s.B.DEV_BAD_SLOT and np.all(sel[1] == -1) and not out[1].any()
    for b in (0, 2):
        assert np.array_equal(sel[b], good_sel[b])
        _close(out[b], good[b])                       # the split over the GPU is another one
    cu = s.torch.tensor([0, 1, 2, 3], dtype=s.torch.int32, device="cuda")
    before = s.bounds.clone()
    s.L.cache.dev_status.zero_()
    s.B.update_page_bounds(s.L.cache.desc, 3, slot, s.L.seq_len, cu, 1, s.bounds, s.exponents)
    assert s.L.cache.status() == s.B.DEV_BAD_SLOT and s.torch.equal(before, s.bounds)
    # an entry that is no page: it is the last choice, and skipped when it is chosen all the same
    s.L.cache.dev_status.zero_()
    victim = int(good_sel[0, 0, 0])
    s.L.cache.page_table[0, victim] = -7
    sel, out = s.sparse(Q, 4)
    assert s.L.cache.status() == s.B.DEV_BAD_PAGE_ID and victim not in sel[0, 0].tolist()
    for b in (1, 2):
        _close(out[b], good[b])
    # a sequence longer than promised: pages beyond the promise are no candidates
    s.L.cache.dev_status.zero_()
    sel, _ = s.sparse(Q, 4, max_seq_len=700)
    assert s.L.cache.status() & s.B.DEV_BAD_COUNT and sel[1:].max() < 11


def test_nan_bounds_fields_and_damaged_tokens_stay_local():
    """A key that is not a number leaves the page's bounds to its other tokens."""
    s = Sparse([1000, 1000], 4, 1, 2, seed=18)
    low, up, _ = s.oracle_bounds(0, 0)
    page = int(s.L.cache.page_table[0, 3])
    rec = s.L.cache.pages.view(-1, 1, s.L.cache.page_bytes)[page, 0]
    meta = rec[-512:].view(s.torch.int16).view(4, 8, 2, 4)          # [block][token & 7][token >> 3][step, x_min of keys, of values]
    meta[1, 2, 1, 1] = 0x7E00                                        # token 26's offset: not a number
    s.update([1000, 1000])
    codes, step, zero = s.L.gpu_codes(0, 0, 0)
    keep = np.array([r for r in range(192, 256) if r != 192 + 26])
    ref = S.page_bounds(codes[keep].astype(np.int64), np.stack([step, zero], 1)[keep])
    assert np.array_equal(s.bounds[page, 0].cpu().numpy(), np.stack(ref[:2])) and int(s.exponents[page, 0]) == ref[2]


def test_pages_far_behind_in_a_large_pool():
    """Records, bounds and copies beyond 2^32 bytes of the pool."""
    import torch
    from paper_2609_38121_b200 import binding as B
    n_pages = 130000                                                 # of 36864 bytes: 4.8 GB
    s = Sparse([700, 300], 32, 8, 2, seed=19)
    c = s.L.cache
    small = (c.pages, c.page_table.clone(), s.bounds, s.exponents)
    q, Q = s.queries()
    sel0, out0 = s.sparse(Q, 3)
    big = torch.zeros(n_pages * c.page_bytes, dtype=torch.uint8, device="cuda")
    bounds, exponents = torch.zeros((n_pages, 8, 2, 128), dtype=torch.int8, device="cuda"), torch.zeros((n_pages, 8), dtype=torch.int8, device="cuda")
    n_small = small[0].numel() // c.page_bytes
    shift = n_pages - n_small
    big[:small[0].numel()] = small[0]
    bounds[:n_small], exponents[:n_small] = small[2], small[3]
    c.desc.pages, c.desc.n_pages = big.data_ptr(), n_pages
    ids = torch.arange(n_small, dtype=torch.int32, device="cuda")
    count = torch.tensor([n_small], dtype=torch.int32, device="cuda")
    B.copy_pages(c.desc, n_small, ids, ids + shift, count, bounds, exponents)
    c.page_table += shift
    assert torch.equal(big[shift * c.page_bytes:], small[0]) and torch.equal(bounds[shift:], small[2]) and torch.equal(exponents[shift:], small[3])
    s.bounds, s.exponents = bounds, exponents
    sel, out = s.sparse(Q, 3)
    assert np.array_equal(sel, sel0) and np.array_equal(out, out0) and c.status() == 0
    bounds.zero_()
    s.update([700, 300])
    sel, out = s.sparse(Q, 3)
    assert np.array_equal(sel, sel0) and np.array_equal(out, out0)


@pytest.mark.parametrize("n_q,n_kv,bits", [(8, 1, 2), (2, 1, 4), (6, 2, 3)])
def test_a_million_positions(n_q, n_kv, bits):
    """The longest sequences there may be: 16383 candidate pages, drawn bounds, packed tokens whose keys and values are zero."""
    import torch
    from paper_2609_38121_b200 import binding as B
    rng, longest, n_select = np.random.default_rng(bits), 1 << 20, 700
    T = np.stack([np.linalg.qr(rng.standard_normal((128, 128)))[0] for _ in range(n_kv)]).astype(np.float32)
    c = B.PagedCache(n_q, n_kv, bits, 2, longest, 4, 64, 1, 0.96, 0.92, T, T, page_order=rng.permutation(2 * 16384), page_bounds=True)
    gen = torch.Generator(device="cuda").manual_seed(bits)
    up = torch.randint(20, 127, c.bounds.shape[:2] + (128,), generator=gen, device="cuda", dtype=torch.int32)
    low = -torch.randint(20, 127, up.shape, generator=gen, device="cuda", dtype=torch.int32)
    c.bounds.copy_(torch.stack([low, up], 2))
    c.exponents.copy_(torch.randint(-6, -4, c.exponents.shape, generator=gen, device="cuda"))
    for t in (c.ring_kv, c.sink_kv):
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    lens = [longest, 999_937]
    q = W.bf16_round_f32(rng.standard_normal((2, n_q, 128)).astype(np.float32) * 2)
    Q = torch.from_numpy(W.f32_to_bf16_bits(q).view(np.int16)).cuda()
    slot, seq_len = torch.arange(2, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    sel, out = torch.zeros((2, n_kv, n_select), dtype=torch.int32, device="cuda"), torch.zeros((2, n_q, 128), dtype=torch.bfloat16, device="cuda")
    B.decode_attn_sparse(c.desc, 2, slot, seq_len, longest, Q, c.bounds, c.exponents, n_select, sel, out)
    assert c.status() == 0
    sel, out, table, G = sel.cpu().numpy(), out.float().cpu().numpy().astype(np.float64), c.page_table.cpu().numpy(), n_q // n_kv
    bounds, e = c.bounds.cpu().numpy().astype(int), c.exponents.cpu().numpy().astype(int)
    ring, sink = c.ring_kv.float().cpu().numpy().astype(np.float64), c.sink_kv.float().cpu().numpy().astype(np.float64)
    for b in range(2):
        lo, hi, first, n = S.packed_range(lens[b], 4, 64, 1)
        for h in range(n_kv):
            row = table[b, first:first + n]
            qc = [O.query_compensation(T[h], q[b, h * G + g][None])[0] for g in range(G)]
            assert np.array_equal(sel[b, h], S.select(S.page_keys(qc, bounds[row, h, 0], bounds[row, h, 1], e[row, h], SCALE), n_select, first))
            packed = sum(min(hi, 64 * p + 64) - max(lo, 64 * p) for p in sel[b, h])
            rows = [p % c.ring_cap for p in range(hi, lens[b])]
            K, V = (np.concatenate([sink[b, h, i], ring[b, h, i][rows]]) for i in range(2))
            ref = []
            for x in qc:
                p = np.exp(SCALE * (K @ x))
                ref.append(p @ V / (p.sum() + packed))
            _close(out[b, h * G:(h + 1) * G], np.stack(ref))


def test_captured_steps_and_other_streams():
    """A decode step of append, bounds and sparse attention, captured once and replayed over growing sequences, on a stream of its
    own: the results of the separate calls."""
    import torch
    from paper_2609_38121_b200 import binding as B
    runs = []
    for captured in (False, True):
        s = Sparse([700, 500], 8, 2, 2, seed=20, fill=False)
        s.append([690, 490])
        c, L = s.L.cache, s.L
        K = torch.zeros((2, 2, 128), dtype=torch.int16, device="cuda")
        V, Q = torch.zeros_like(K), torch.zeros((2, 8, 128), dtype=torch.int16, device="cuda")
        cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
        sel = torch.zeros((2, 2, 3), dtype=torch.int32, device="cuda")
        out = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device="cuda")
        need = B.sparse_workspace_bytes(c.desc, 2, 704, 3)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")

        def step(stream=None):
            B.append(c.desc, 2, L.slot, L.seq_len, cu, 2, 1, K, V, stream)
            B.update_page_bounds(c.desc, 2, L.slot, L.seq_len, cu, 1, s.bounds, s.exponents, stream)
            B.decode_attn_sparse(c.desc, 2, L.slot, L.seq_len, 704, Q, s.bounds, s.exponents, 3, sel, out, ws, need, stream=stream)

        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        if captured:
            state = [t.clone() for t in (L.seq_len, c.pages, c.ring_kv, c.sink_kv, s.bounds, s.exponents)]
            stream.wait_stream(torch.cuda.current_stream())
            step(stream)                                             # first calls outside the capture
            stream.synchronize()
            for t, x in zip((L.seq_len, c.pages, c.ring_kv, c.sink_kv, s.bounds, s.exponents), state):
                t.copy_(x)
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                step(stream)
        got = []
        for i in range(10):
            for t, x in ((K, [L.tokens[b][0][L.done[b] + i] for b in range(2)]), (V, [L.tokens[b][1][L.done[b] + i] for b in range(2)]),
                         (Q, [s.wl.queries(b, L.done[b] + i) for b in range(2)])):
                t.copy_(torch.from_numpy(W.f32_to_bf16_bits(np.stack(x)).view(np.int16)))
            torch.cuda.synchronize()
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            got.append((sel.cpu().numpy(), out.float().cpu().numpy(), s.bounds.cpu().numpy()))
        assert c.status() == 0
        runs.append(got)
    for a, b in zip(*runs):
        for x, y in zip(a, b):
            assert np.array_equal(x, y)


def test_two_calls_at_once_and_repeated_calls_agree():
    import torch
    s = Sparse([5000, 3000, 100], 16, 2, 4, seed=21)
    q, Q = s.queries()
    want = s.sparse(Q, 12)
    streams = [torch.cuda.Stream() for _ in range(2)]
    c, B = s.L.cache.desc, s.B
    need = B.sparse_workspace_bytes(c, 3, s.L.max_seq_len, 12)
    bufs = [(torch.empty((3, 2, 12), dtype=torch.int32, device="cuda"), torch.empty((3, 16, 128), dtype=torch.bfloat16, device="cuda"),
             torch.empty(need, dtype=torch.uint8, device="cuda")) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (sel, out, ws) in zip(streams, bufs):
            B.decode_attn_sparse(c, 3, s.L.slot, s.L.seq_len, s.L.max_seq_len, Q, s.bounds, s.exponents, 12, sel, out, ws, need, stream=st)
    torch.cuda.synchronize()
    for sel, out, _ in bufs:
        assert np.array_equal(sel.cpu().numpy(), want[0]) and np.array_equal(out.float().cpu().numpy(), want[1])
