"""Host-side refusals of the K/V cache's calls and of its attention, and the oracle's
bookkeeping: no GPU. Only calls that return before any CUDA call are made."""
import ctypes as C

import numpy as np
import pytest

from oracle.kvcache import Cache
from paper_2608_11742_gb300 import rps

P = 1 << 20  # a 16-byte aligned address that is never read: every call here is refused


def cache(**kw):
    base = dict(k=P, v=P, dtype=rps.RPS_BF16, n_layers=2, n_pages=10, n_heads=4, page_size=16, head_dim=128,
                layer_stride=10 * 4 * 16 * 128, page_stride=4 * 16 * 128, head_stride=16 * 128, token_stride=128,
                page_ref=P, table=P, len=P, n_req=2, n_branch=3, max_pages=5)
    base.update(kw)
    return rps.RpsKvCache(**base)


INVALID = [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(dtype=rps.RPS_F32), dict(dtype=7),
           dict(n_layers=0), dict(n_pages=0), dict(n_heads=0), dict(page_size=0), dict(page_stride=7),
           dict(head_stride=100), dict(token_stride=-128), dict(layer_stride=0)]
UNSUPPORTED = [dict(head_dim=64), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(n_layers=1025),
               dict(n_heads=1025)]
BOOK_INVALID = [dict(page_ref=None), dict(table=None), dict(len=None), dict(n_req=0), dict(n_branch=0), dict(max_pages=0)]
BOOK_UNSUPPORTED = [dict(n_req=1 << 19), dict(max_pages=1 << 27), dict(n_pages=1 << 30)]


def calls(lib, kv):
    at, big = C.addressof(kv), 1 << 40
    return {
        "reorder": lambda: lib.rps_kv_reorder(at, P, None, P, big, None),
        "fork": lambda: lib.rps_kv_fork_branches(at, P, None, P, big, None),
        "commit": lambda: lib.rps_kv_commit(at, P, P, big, None),
        "resize": lambda: lib.rps_kv_resize(at, P, P, big, None),
        "compact": lambda: lib.rps_kv_compact(at, None, P, big, None),
        "write": lambda: lib.rps_kv_write(at, 0, P, P, 1, 512, 512, 128, None),
    }


@pytest.mark.parametrize("kw,status", [(k, rps.RPS_ERR_INVALID_ARG) for k in INVALID + BOOK_INVALID]
                         + [(k, rps.RPS_ERR_UNSUPPORTED) for k in UNSUPPORTED + BOOK_UNSUPPORTED])
def test_caches_that_are_refused(kw, status):
    kv = cache(**kw)
    assert rps._lib.rps_kv_workspace_bytes(C.addressof(kv)) == 0
    for name, call in calls(rps._lib, kv).items():
        assert call() == status, (name, kw)
    if kw in INVALID + UNSUPPORTED:
        good = cache()
        for a, b in ((kv, good), (good, kv)):
            assert rps._lib.rps_kv_copy_pages(C.addressof(a), C.addressof(b), P, P, 1, None) == status


def test_arguments_that_are_refused():
    lib, bad = rps._lib, rps.RPS_ERR_INVALID_ARG
    kv = cache()
    at, need = C.addressof(kv), lib.rps_kv_workspace_bytes(C.addressof(kv))
    assert need > 0
    for ws, size in ((None, need), (P, need - 1), (P + 8, need)):
        assert lib.rps_kv_reorder(at, P, None, ws, size, None) == bad
        assert lib.rps_kv_resize(at, P, ws, size, None) == bad
        assert lib.rps_kv_commit(at, P, ws, size, None) == bad
        assert lib.rps_kv_fork_branches(at, P, P, ws, size, None) == bad
        assert lib.rps_kv_compact(at, P, ws, size, None) == bad
    assert lib.rps_kv_reorder(at, None, None, P, need, None) == bad
    assert lib.rps_kv_resize(at, None, P, need, None) == bad
    assert lib.rps_kv_commit(at, None, P, need, None) == bad
    assert lib.rps_kv_fork_branches(at, None, P, P, need, None) == bad
    assert lib.rps_kv_fork_branches(C.addressof(cache(n_branch=1)), P, P, P, need, None) == bad
    assert lib.rps_kv_fork_branches(None, P, P, P, need, None) == bad
    assert lib.rps_kv_compact(None, P, P, need, None) == bad
    for other in (dict(dtype=rps.RPS_F16), dict(n_layers=1), dict(n_heads=2), dict(page_size=32)):
        assert lib.rps_kv_copy_pages(at, C.addressof(cache(**other)), P, P, 1, None) == bad
    assert lib.rps_kv_copy_pages(at, at, None, P, 1, None) == bad
    assert lib.rps_kv_copy_pages(at, at, P, None, 1, None) == bad
    assert lib.rps_kv_copy_pages(at, at, P, P, -1, None) == bad
    assert lib.rps_kv_copy_pages(at, at, P, P, 0, None) == rps.RPS_OK  # nothing to do, nothing enqueued
    write = lambda layer=0, k=P, v=P, n=1, s=512, t=512, h=128: lib.rps_kv_write(at, layer, k, v, n, s, t, h, None)
    for kw in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(k=P + 4), dict(n=0), dict(s=4), dict(t=-8),
               dict(h=1)):
        assert write(**kw) == bad, kw
    assert write(n=1 << 29) == rps.RPS_ERR_UNSUPPORTED


def test_workspace_grows_with_each_size():
    size = lambda **kw: rps._lib.rps_kv_workspace_bytes(C.addressof(cache(**kw)))
    base = size()
    assert size(n_pages=1000) > base and size(n_req=50) > base and size(max_pages=500) > base


def test_oracle_keeps_counts_and_order():
    """Counts are the table's entries; pages go out lowest first; a page given back is taken again first."""
    c = Cache(np.zeros(8), np.full((3, 4), -1), [-1, -1, -1], 16)
    c.resize([33, -1, 16])
    assert c.table[0, :3].tolist() == [0, 1, 2] and c.table[2, 0] == 3
    c.reorder([0, 0, 2], [40, 20, 16])
    assert c.length.tolist() == [33, 20, 16] and c.ref.tolist() == [2, 2, 1, 1, 0, 0, 0, 0]
    c.resize([33, 40, -1])  # the shared second page is copied; the third sequence's page comes back first
    assert c.table[1, :3].tolist() == [0, 3, 4] and c.ref.tolist() == [2, 1, 1, 1, 1, 0, 0, 0]
    c.resize([-1, 40, -1])
    assert c.compact() == 3 and c.table[1, :3].tolist() == [0, 1, 2] and c.err == 0


def attention(**kw):
    base = dict(q=P, out=P, lse=None, n_q=2, n_heads=8, layer=0, causal=0, q_req_stride=6 * 8 * 128, q_token_stride=1024,
                q_head_stride=128, out_req_stride=6 * 8 * 128, out_token_stride=1024, out_head_stride=128,
                shared_len=None, scale=0.1)
    base.update(kw)
    return rps.RpsPrefixAttention(**base)


def test_attention_arguments_that_are_refused():
    lib, good = rps._lib, cache()
    need = lib.rps_prefix_attention_workspace_bytes(C.addressof(good), 2, 8)
    assert need > 0
    call = lambda a, kv=good, ws=P, n=need: lib.rps_prefix_attention_fwd(C.addressof(a), C.addressof(kv), ws, n, None)
    for kw in (dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 2), dict(n_q=0), dict(n_heads=0), dict(n_heads=6),
               dict(layer=2), dict(layer=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(q_head_stride=4), dict(q_token_stride=0), dict(out_req_stride=-8), dict(out_token_stride=100)):
        assert call(attention(**kw)) == rps.RPS_ERR_INVALID_ARG, kw
    for kw in (dict(n_heads=4 * 129), dict(n_q=1 << 28)):
        assert call(attention(**kw)) == rps.RPS_ERR_UNSUPPORTED, kw
    for ws, n in ((None, need), (P + 4, need), (P, need - 1)):
        assert call(attention(), ws=ws, n=n) == rps.RPS_ERR_INVALID_ARG
    for kw in INVALID + BOOK_INVALID:
        assert call(attention(), cache(**kw)) == rps.RPS_ERR_INVALID_ARG, kw
    for kw in UNSUPPORTED + BOOK_UNSUPPORTED:
        assert call(attention(), cache(**kw)) == rps.RPS_ERR_UNSUPPORTED, kw
        assert lib.rps_prefix_attention_workspace_bytes(C.addressof(cache(**kw)), 2, 8) == 0
    assert lib.rps_prefix_attention_fwd(None, C.addressof(good), P, need, None) == rps.RPS_ERR_INVALID_ARG
    assert lib.rps_prefix_attention_fwd(C.addressof(attention()), None, P, need, None) == rps.RPS_ERR_INVALID_ARG
