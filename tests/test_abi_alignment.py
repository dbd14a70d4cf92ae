"""Arrays of 32-bit integers that are not aligned to 4 bytes are refused on the host, by every call that hands them to a kernel (no
GPU needed: nothing is launched)."""
import ctypes as C

import pytest

from paper_2609_38121_b200 import binding as B
from tests import test_abi_sparse as S

P, BIG = S.P, 1 << 30
PROLOGUE = C.byref(B.wushkv_prologue(P, 64, 0, None, None, 0.0))
APPEND = dict(cache=S._cache(), batch=2, slot=P, seq_len=P, cu_new=P, total_new=4, max_new=2, K=P, V=P)
DECODE = dict(cache=S._cache(), batch=2, slot=P, seq_len=P, max_seq_len=1000, Q=P, O=P, ws=P, ws_bytes=BIG)
PREFILL = dict(cache=S._cache(), batch=2, slot=P, seq_len=P, cu_new=P, total_new=4, max_new=2, K=P, V=P, Q=P, O=P, ws=P, ws_bytes=BIG)
STEP = dict(cache=S._cache(), batch=2, slot=P, seq_len=P, cu_new=P, max_seq_len=1000, K=P, V=P, Q=P, O=P, ws=P, ws_bytes=BIG)


def _with(args, before):
    """The arguments with a prologue ahead of one of them."""
    return {k: v for name, value in args.items() for k, v in (([("prologue", PROLOGUE)] if name == before else []) + [(name, value)])}


CALLS = [
    (B.lib.wushkv_append, APPEND, ("slot", "seq_len", "cu_new")),
    (B.lib.wushkv_append_projected, {**APPEND, "prologue": PROLOGUE}, ("slot", "seq_len", "cu_new")),
    (B.lib.wushkv_decode_attn, DECODE, ("slot", "seq_len")),
    (B.lib.wushkv_decode_attn_projected, _with(DECODE, "O"), ("slot", "seq_len")),
    (B.lib.wushkv_decode_step, STEP, ("slot", "seq_len", "cu_new")),
    (B.lib.wushkv_prefill_attn, PREFILL, ("slot", "seq_len", "cu_new")),
    (B.lib.wushkv_prefill_attn_projected, _with(PREFILL, "O"), ("slot", "seq_len", "cu_new")),
    (B.lib.wushkv_update_page_bounds, S.BOUNDS, ("slot", "seq_len", "cu_new")),
    (B.lib.wushkv_select_pages, S.SELECT, ("slot", "seq_len", "selected")),
    (B.lib.wushkv_decode_attn_selected, S.ATTEND, ("slot", "seq_len", "selected")),
    (B.lib.wushkv_decode_attn_sparse, S.SPARSE, ("slot", "seq_len", "selected")),
    (B.lib.wushkv_pages_reserve, S.RESERVE, ("slot", "seq_len", "cu_new", "copy_src", "copy_dst", "n_copies", "ws")),
    (B.lib.wushkv_pages_fork, S.FORK, ("src", "dst", "src_len")),
    (B.lib.wushkv_pages_release, S.RELEASE, ("slot", "keep")),
    (B.lib.wushkv_pages_compact, S.COMPACT, ("copy_src", "copy_dst", "n_copies", "n_live", "ws")),
    (B.lib.wushkv_copy_pages, S.COPY_PAGES, ("src", "dst", "n_copies")),
    (B.lib.wushkv_copy_windows, S.COPY_WINDOWS, ("src", "dst", "src_len")),
]


@pytest.mark.parametrize("fn,args,names", CALLS, ids=[c[0].__name__ for c in CALLS])
def test_unaligned_integers_are_refused(fn, args, names):
    for name in names:
        for off in (1, 2, 3):
            assert fn(*{**args, name: P + off}.values(), None) == B.EINVAL, (name, off)
