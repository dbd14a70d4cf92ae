"""Refusals of the sparse-attention and page-pool entry points, made on the host before anything is launched (no GPU needed),
and the layout of wushkv_page_pool."""
import ctypes as C
import os
import re

import pytest

from paper_2609_38121_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096            # a well-aligned address that nothing reads


def _cache(**kw):
    base = dict(n_q=8, n_kv=2, d=128, bits=2, page_tokens=64, s_sink=4, s_keep=64, s_flush=1, boundary_lag=0, n_slots=2, max_pages=16, ring_cap=64,
                kappa_k=0.96, kappa_v=0.92, sm_scale=0.1, quantizer=0, n_pages=32, pages=P, page_table=P, sink_kv=P, ring_kv=P, T_K=P, T_K_invT=P, dev_status=P)
    return C.byref(B.wushkv_cache(**{**base, **kw}))


def _pool(**kw):
    return C.byref(B.wushkv_page_pool(**{**dict(n_slots=2, max_pages=16, n_pages=32, page_table=P, refs=P, dev_status=P), **kw}))


def test_pool_layout_matches_the_header():
    text = open(os.path.join(ROOT, "include", "wushkv.h")).read()
    body = re.search(r"typedef struct wushkv_page_pool \{(.*?)\} wushkv_page_pool;", text, flags=re.S).group(1)
    names = [re.findall(r"[A-Za-z_][A-Za-z_0-9]*", part)[-1] for decl in body.split(";") if decl.strip() for part in decl.split(",")]
    assert names == [f[0] for f in B.wushkv_page_pool._fields_]
    assert C.sizeof(B.wushkv_page_pool) == 2 * 4 + 8 + 3 * 8


BOUNDS = dict(cache=_cache(), batch=2, slot=P, seq_len=P, cu_new=P, max_new=5, bounds=P, exponents=P)
SELECT = dict(cache=_cache(), batch=2, slot=P, seq_len=P, max_seq_len=1000, Q=P, prologue=None, bounds=P, exponents=P, n_select=4, selected=P)
ATTEND = dict(cache=_cache(), batch=2, slot=P, seq_len=P, max_seq_len=1000, Q=P, prologue=None, selected=P, n_select=4, O=P)
SPARSE = dict(cache=_cache(), batch=2, slot=P, seq_len=P, max_seq_len=1000, Q=P, prologue=None, bounds=P, exponents=P, n_select=4, selected=P, O=P, ws=P,
              ws_bytes=1 << 30)
RESERVE = dict(pool=_pool(), batch=2, slot=P, seq_len=P, cu_new=P, copy_src=P, copy_dst=P, n_copies=P, ws=P, ws_bytes=1 << 20)
FORK = dict(pool=_pool(), n=2, src=P, dst=P, src_len=P)
RELEASE = dict(pool=_pool(), n=2, slot=P, keep=None)
COMPACT = dict(pool=_pool(), copy_src=P, copy_dst=P, n_copies=P, n_live=P, ws=P, ws_bytes=1 << 20)
COPY_PAGES = dict(cache=_cache(), max_copies=3, src=P, dst=P, n_copies=P, bounds=P, exponents=P)
COPY_WINDOWS = dict(cache=_cache(), n=2, src=P, dst=P, src_len=P)

REFUSED = [
    (B.lib.wushkv_update_page_bounds, BOUNDS, dict(cache=[None, _cache(bits=5), _cache(d=64), _cache(n_q=9), _cache(pages=None)], batch=[0, -1, 65536], slot=[None],
                                                   seq_len=[None], cu_new=[None], max_new=[-1], bounds=[None, P + 8], exponents=[None])),
    (B.lib.wushkv_select_pages, SELECT, dict(cache=[None, _cache(n_kv=0)], batch=[0, 65536], slot=[None], seq_len=[None], max_seq_len=[0, -5], Q=[None, P + 2],
                                             bounds=[None, P + 1], exponents=[None], n_select=[0, -1, (1 << 30) + 1], selected=[None], prologue=[C.byref(B.wushkv_prologue())])),
    (B.lib.wushkv_decode_attn_selected, ATTEND, dict(cache=[None], batch=[0, 65536], slot=[None], seq_len=[None], max_seq_len=[0], Q=[None, P + 8], selected=[None],
                                                     n_select=[0, (1 << 30) + 1], O=[None, P + 2], prologue=[C.byref(B.wushkv_prologue())])),
    (B.lib.wushkv_decode_attn_sparse, SPARSE, dict(cache=[None], batch=[0, 65536], bounds=[None, P + 4], exponents=[None], n_select=[0, (1 << 30) + 1], O=[None, P + 8])),
    (B.lib.wushkv_decode_attn_sparse, {**SPARSE, "selected": None}, dict(cache=[None, _cache(bits=1)], batch=[0], n_select=[0], max_seq_len=[0], ws=[None, P + 128])),
    (B.lib.wushkv_pages_reserve, RESERVE, dict(pool=[None, _pool(n_pages=0), _pool(n_slots=0), _pool(max_pages=-1), _pool(refs=None), _pool(page_table=P + 2),
                                                     _pool(dev_status=None), _pool(n_pages=1 << 31), _pool(n_pages=(1 << 30) + 1), _pool(max_pages=(1 << 20) + 1)], batch=[0, -2, (1 << 30) + 1], slot=[None], seq_len=[None], cu_new=[None],
                                               copy_src=[None], copy_dst=[None], n_copies=[None], ws=[None, P + 1])),
    (B.lib.wushkv_pages_fork, FORK, dict(pool=[None], n=[-1], src=[None], dst=[None], src_len=[None])),
    (B.lib.wushkv_pages_release, RELEASE, dict(pool=[None], n=[-1], slot=[None])),
    (B.lib.wushkv_pages_compact, COMPACT, dict(pool=[None], copy_src=[None], copy_dst=[None], n_copies=[None], n_live=[None], ws=[None])),
    (B.lib.wushkv_copy_pages, COPY_PAGES, dict(cache=[None], max_copies=[-1], src=[None], dst=[None], n_copies=[None], bounds=[None, P + 2], exponents=[None])),
    (B.lib.wushkv_copy_windows, COPY_WINDOWS, dict(cache=[None], n=[-1, 65536], src=[None], dst=[None], src_len=[None])),
]


@pytest.mark.parametrize("fn,good,bad", REFUSED, ids=["%s-%d" % (f[0].__name__, k) for k, f in enumerate(REFUSED)])
def test_bad_arguments_are_refused(fn, good, bad):
    for name, values in bad.items():
        for value in values:
            assert fn(*{**good, name: value}.values(), None) == B.EINVAL, (name, value)


def test_capacities():
    assert B.lib.wushkv_decode_attn_sparse(*{**SPARSE, "selected": None, "ws_bytes": 100}.values(), None) == B.ECAPACITY
    assert B.lib.wushkv_pages_reserve(*{**RESERVE, "ws_bytes": 100}.values(), None) == B.ECAPACITY
    assert B.lib.wushkv_pages_compact(*{**COMPACT, "ws_bytes": 4 * 3 * 32 - 1}.values(), None) == B.ECAPACITY
    # more candidate pages than the selection ranks
    assert B.lib.wushkv_select_pages(*{**SELECT, "max_seq_len": (1 << 20) + 1000}.values(), None) == B.ECAPACITY
    assert B.lib.wushkv_decode_attn_sparse(*{**SPARSE, "max_seq_len": (1 << 20) + 1000}.values(), None) == B.ECAPACITY
    # the recent window does not fit into the ring
    assert B.lib.wushkv_copy_windows(*{**COPY_WINDOWS, "cache": _cache(ring_cap=63)}.values(), None) == B.ECAPACITY


def test_nothing_to_do_is_fine():
    assert B.lib.wushkv_update_page_bounds(*{**BOUNDS, "max_new": 0}.values(), None) == B.OK
    assert B.lib.wushkv_pages_fork(*{**FORK, "n": 0}.values(), None) == B.OK
    assert B.lib.wushkv_pages_release(*{**RELEASE, "n": 0}.values(), None) == B.OK
    assert B.lib.wushkv_copy_pages(*{**COPY_PAGES, "max_copies": 0}.values(), None) == B.OK
    assert B.lib.wushkv_copy_windows(*{**COPY_WINDOWS, "n": 0}.values(), None) == B.OK


def test_workspace_sizes():
    def sparse(batch, longest, n, **kw):
        return B.lib.wushkv_sparse_workspace_bytes(_cache(**kw), batch, longest, n)
    assert sparse(0, 100, 4) == 0 and sparse(2, 0, 4) == 0 and sparse(2, 100, 0) == 0 and sparse(2, 100, 4, bits=7) == 0
    assert sparse(2, 1000, 5) >= 2 * 2 * 5 * 4 and sparse(100, 1000, 4) >= 100 * 2 * 4 * 4
    assert B.lib.wushkv_pages_workspace_bytes(_pool(), 0) == 0 and B.lib.wushkv_pages_workspace_bytes(_pool(n_pages=-1), 4) == 0
    assert B.lib.wushkv_pages_workspace_bytes(_pool(), 4) >= 3 * 32 * 4
    assert B.lib.wushkv_pages_workspace_bytes(_pool(), 1000) >= 3 * 1000 * 4
