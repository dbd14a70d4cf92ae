"""Oracle of the sparse decode attention (bounds of packed pages, selection of pages, attention over them) and of the page
pool, in float64 / plain integers, written from the definitions in the header; no code in common with the library."""
from __future__ import annotations

import math

import numpy as np

from oracle import wushkv_oracle as O

PAGE = 64


# --------------------------------------------------------------------------
# bounds and selection
# --------------------------------------------------------------------------


def page_bounds(codes, meta):
    """Bounds of one page and head from its existing tokens: codes [n][d] integers, meta [n][2] = (step, x_min) as stored.
    Returns (lower, upper) int arrays [d] and the exponent e."""
    khat = np.float32(meta[:, 1:2] + meta[:, 0:1] * codes.astype(np.float64)).astype(np.float64)
    up, low = khat.max(axis=0), khat.min(axis=0)
    most = max(np.abs(up).max(), np.abs(low).max())
    e = -31
    while most > 127 * 2.0 ** e:
        e += 1
    return np.floor(low / 2.0 ** e).astype(int), np.ceil(up / 2.0 ** e).astype(int), e


def fixed_point(q):
    """The 16-bit fixed-point query and its unit: q ~ unit * integers."""
    most = np.abs(q).max()
    if not (most > 0 and most < 3e38):
        return np.zeros(q.shape), 0.0
    return np.rint(q * (32512.0 / most)), most / 32512.0


def page_scores(q, lower, upper, e, sm_scale):
    """Scores of all pages for one compensated query: lower, upper [pages][d], e [pages]; float32."""
    qi, unit = fixed_point(q)
    dot = np.maximum(qi, 0) @ upper.T.astype(np.float64) + np.minimum(qi, 0) @ lower.T.astype(np.float64)
    assert np.all(np.abs(dot) < 2.0 ** 31)
    return np.float32(dot) * np.float32(2.0) ** np.asarray(e).astype(np.float32) * np.float32(unit * float(np.float32(sm_scale)))


def page_keys(queries, lower, upper, e, sm_scale):
    """Keys of all pages for the query heads of a group: how far the page is below the best page of the head it matters most to."""
    scores = np.stack([page_scores(q, lower, upper, e, sm_scale) for q in queries])
    return (scores - scores.max(axis=1, keepdims=True)).max(axis=0)


def select(keys, n_select, first=0):
    """The n_select largest keys, ties to the lower index, ascending, -1 behind them."""
    order = sorted(range(len(keys)), key=lambda p: (-float(keys[p]), p))[:n_select]
    out = np.full(n_select, -1, dtype=np.int64)
    out[:len(order)] = np.sort(np.asarray(order, dtype=np.int64)) + first
    return out


def packed_range(S, s_sink, s_keep, s_flush, lag=0):
    """Packed positions [lo, hi) and the page indexes [first, first + n) that hold them."""
    nq = O.n_quantized(S - lag, s_sink, s_keep, s_flush)
    lo, hi = s_sink, s_sink + nq
    first = lo // PAGE
    return lo, hi, first, ((hi - 1) // PAGE - first + 1 if nq > 0 else 0)


def sparse_attention(q_comp, K_eff, V_eff, lo, hi, pages, sm_scale):
    """Attention of one compensated query over the windows and the listed pages (page indexes; -1 ignored).  K_eff / V_eff are
    the rows that dense attention reads ([S][d]); [lo, hi) the packed positions."""
    keep = np.ones(len(K_eff), dtype=bool)
    keep[lo:hi] = False
    for p in pages:
        if p >= 0:
            keep[max(lo, p * PAGE):min(hi, (p + 1) * PAGE)] = True
    if not keep.any():
        return np.zeros(V_eff.shape[1])
    return O.attention_one_query(q_comp, K_eff[keep], V_eff[keep], sm_scale)


# --------------------------------------------------------------------------
# the page pool: one request after the other
# --------------------------------------------------------------------------


class Pool:
    """Page table and counts; the same calls as the library's, carried out in order."""

    def __init__(self, n_slots, max_pages, n_pages):
        self.table = np.full((n_slots, max_pages), -1, dtype=np.int64)
        self.refs = np.zeros(n_pages, dtype=np.int64)
        self.empty = False

    def _drop(self, entry):
        if entry != -1:
            self.refs[entry if entry >= 0 else -2 - entry] -= 1

    def _free(self):
        return [p for p in range(len(self.refs)) if self.refs[p] == 0]

    def reserve(self, requests):
        """requests: (slot, length, new tokens).  Returns the copies as (source, destination) pairs."""
        for slot, length, new in requests:                         # tokens behind the table's end: nothing, a shared last page is locked
            if new > 0 and (length + new - 1) // PAGE >= self.table.shape[1] and length % PAGE and length // PAGE < self.table.shape[1]:
                e = self.table[slot, length // PAGE]
                page = e if e >= 0 else -2 - e
                if e != -1 and self.refs[page] > 1:
                    self.table[slot, length // PAGE] = -2 - page
        table, refs, free, copies, enough = self.table.copy(), self.refs.copy(), self._free(), [], True
        for slot, length, new in requests:
            if new <= 0 or (length + new - 1) // PAGE >= table.shape[1]:
                continue
            for i in range(length // PAGE, (length + new - 1) // PAGE + 1):
                e = table[slot, i]
                page = e if e >= 0 else -2 - e
                if e != -1 and refs[page] == 1:
                    table[slot, i] = page
                    continue
                if not free:
                    enough = False
                    break
                own = free.pop(0)
                if e != -1:
                    if i * PAGE < length:
                        copies.append((page, own))
                    refs[page] -= 1
                table[slot, i] = own
                refs[own] = 1
        if enough:
            self.table, self.refs = table, refs
            return copies
        self.empty = True
        for slot, length, new in requests:
            if new <= 0 or (length + new - 1) // PAGE >= table.shape[1]:
                continue
            for i in range(length // PAGE, (length + new - 1) // PAGE + 1):
                e = self.table[slot, i]
                if e != -1:
                    page = e if e >= 0 else -2 - e
                    self.table[slot, i] = -2 - page if self.refs[page] > 1 else page
        return []

    def fork(self, src, dst, length):
        for i in range(self.table.shape[1]):
            old, e = self.table[dst, i], self.table[src, i]
            new = -1
            if i * PAGE < length:
                new = e if e >= 0 else -2 - e
                self.refs[new] += 1
            self._drop(old)
            self.table[dst, i] = new

    def release(self, slot, keep=0):
        for i in range(math.ceil(max(keep, 0) / PAGE), self.table.shape[1]):
            self._drop(self.table[slot, i])
            self.table[slot, i] = -1

    def compact(self):
        """Returns the copies and the number of live pages."""
        live = int((self.refs > 0).sum())
        moves = list(zip([p for p in range(live, len(self.refs)) if self.refs[p] > 0], [p for p in range(live) if self.refs[p] == 0]))
        where = {a: b for a, b in moves}
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        for s in range(self.table.shape[0]):
            for i in range(self.table.shape[1]):
                e = self.table[s, i]
                if e >= 0:
                    self.table[s, i] = where.get(e, e)
                elif e < -1:
                    self.table[s, i] = -2 - where.get(-2 - e, -2 - e)
        return moves, live

    def check(self):
        """The counts are the numbers of entries that name the pages."""
        named = np.zeros(len(self.refs), dtype=np.int64)
        for e in self.table.reshape(-1):
            if e != -1:
                named[e if e >= 0 else -2 - e] += 1
        assert np.array_equal(named, self.refs)
