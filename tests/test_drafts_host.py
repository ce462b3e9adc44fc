"""Host-side refusals of positions, norms, appending and drafted tokens, the frequencies in
turns, and the oracle of drafted tokens: no GPU. Only calls that return before any CUDA call are made."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import drafts
from oracle.kvcache import Cache
from paper_2608_11742_gb300 import rps
from test_kvcache_host import BOOK_INVALID, BOOK_UNSUPPORTED, INVALID, UNSUPPORTED, P, cache

BAD, BEYOND = rps.RPS_ERR_INVALID_ARG, rps.RPS_ERR_UNSUPPORTED
LIB = rps._lib


def rope(**kw):
    base = dict(turns=P, rotary_dim=128, interleaved=0, amplitude=1.0, eps=1e-6, q_weight=P, k_weight=P)
    return rps.RpsRope(**{**base, **kw})


def heads(n=4, **kw):
    base = dict(src=P, dst=P, n_heads=n, src_seq=8 * 4 * 128, src_token=512, src_head=128, dst_seq=8 * 4 * 128, dst_token=512,
                dst_head=128)
    return rps.RpsHeads(**{**base, **kw})


def at(x):
    return None if x is None else C.addressof(x)


ROPES = [(dict(turns=None), BAD), (dict(turns=P + 4), BAD), (dict(rotary_dim=-16), BAD), (dict(rotary_dim=24), BEYOND),
         (dict(rotary_dim=144), BAD), (dict(amplitude=float("nan")), BAD), (dict(amplitude=float("inf")), BAD),
         (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(q_weight=P + 2), BAD), (dict(k_weight=P + 8), BAD)]
HEADS = [(dict(src=None), BAD), (dict(src=P + 8), BAD), (dict(n_heads=0), BAD), (dict(n_heads=1 << 20), BEYOND),
         (dict(src_seq=-8), BAD), (dict(src_token=4), BAD), (dict(src_head=100), BAD)]
DSTS = [(dict(dst=None), BAD), (dict(dst=P + 4), BAD), (dict(dst_seq=0), BAD), (dict(dst_token=-512), BAD), (dict(dst_head=12), BAD)]


@pytest.mark.parametrize("kw,status", ROPES)
def test_ropes_that_are_refused(kw, status):
    r, h, kv = rope(**kw), heads(), cache()
    assert LIB.rps_rope_heads(at(r), at(h), at(h), rps.RPS_BF16, 128, 2, 8, P, None) == status
    assert LIB.rps_kv_append(at(kv), 0, at(r), None, at(h), at(h), 8, None, None, None) == status


@pytest.mark.parametrize("kw,status", HEADS + DSTS)
def test_heads_that_are_refused(kw, status):
    r, h, good, kv = rope(), heads(**kw), heads(), cache()
    for q, k in ((h, good), (good, h), (h, None)):
        assert LIB.rps_rope_heads(at(r), at(q), at(k), rps.RPS_F16, 128, 2, 8, None, None) == status
    assert LIB.rps_kv_append(at(kv), 0, at(r), at(h), at(good), at(good), 8, None, None, None) == status
    if (kw, status) in HEADS:
        expect = BAD if "n_heads" in kw else status  # (not the cache's number of heads)
        for k, v in ((h, good), (good, h)):
            assert LIB.rps_kv_append(at(kv), 0, at(r), None, at(k), at(v), 8, None, None, None) == expect


def test_arguments_of_rope_heads_that_are_refused():
    r, h = rope(), heads()
    call = lambda r=r, q=h, dtype=rps.RPS_BF16, d=128, n_seq=2, n_tok=8: LIB.rps_rope_heads(at(r), at(q), None, dtype, d, n_seq,
                                                                                         n_tok, P, None)
    for kw, status in ((dict(r=None), BAD), (dict(q=None), BAD), (dict(dtype=rps.RPS_F32), BAD), (dict(dtype=9), BAD),
                       (dict(d=0), BAD), (dict(d=24), BEYOND), (dict(d=272), BEYOND), (dict(n_seq=0), BAD), (dict(n_tok=-1), BAD),
                       (dict(d=64), BAD)):
        assert call(**kw) == status, kw


@pytest.mark.parametrize("kw,status", [(k, BAD) for k in INVALID + BOOK_INVALID] + [(k, BEYOND) for k in UNSUPPORTED + BOOK_UNSUPPORTED])
def test_caches_that_are_refused(kw, status):
    kv, r, h = cache(**kw), rope(), heads(kw.get("n_heads", 4) or 4)
    a = attention()
    assert LIB.rps_kv_append(at(kv), 0, at(r), None, at(h), at(h), 8, None, None, None) == status
    assert LIB.rps_kv_keep_path(at(kv), P, P, 4, None, 8, P, None) == status
    assert LIB.rps_tree_attention_workspace_bytes(at(kv), 8, 4) == 0
    assert LIB.rps_tree_attention_fwd(at(a), at(kv), P, 1 << 40, None) == status


def attention(**kw):
    base = dict(q=P, out=P, lse=P, n_q=8, n_heads=4, layer=0, q_seq_stride=8 * 512, q_token_stride=512, q_head_stride=128,
                out_seq_stride=8 * 512, out_token_stride=512, out_head_stride=128, n_tok=P, mask=P, scale=0.1)
    return rps.RpsTreeAttention(**{**base, **kw})


def test_arguments_that_are_refused():
    kv, r, h = cache(), rope(), heads()
    append = lambda layer=0, k=h, v=h, n=8: LIB.rps_kv_append(at(kv), layer, at(r), None, at(k), at(v), n, None, None, None)
    for kw in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(n=0), dict(k=heads(2)), dict(v=heads(5))):
        assert append(**kw) == BAD, kw
    masks = lambda parent=P, n_seq=2, n=8, mask=P: LIB.rps_tree_masks(parent, None, None, n_seq, n, mask, None, None)
    for kw, status in ((dict(parent=None), BAD), (dict(mask=None), BAD), (dict(n_seq=0), BAD), (dict(n=0), BAD),
                       (dict(n=rps.RPS_TREE_MAX_TOKENS + 1), BEYOND)):
        assert masks(**kw) == status, kw
    keep = lambda path=P, n_keep=P, n_path=4, n_q=8: LIB.rps_kv_keep_path(at(kv), path, n_keep, n_path, None, n_q, None, None)
    for kw, status in ((dict(path=None), BAD), (dict(n_keep=None), BAD), (dict(n_path=0), BAD), (dict(n_q=0), BAD),
                       (dict(n_path=1025), BEYOND), (dict(n_q=1025), BEYOND)):
        assert keep(**kw) == status, kw
    many = cache(n_req=1 << 16, n_branch=1)
    assert LIB.rps_kv_keep_path(at(many), P, P, 4, None, 8, None, None) == BEYOND
    need = LIB.rps_tree_attention_workspace_bytes(at(kv), 8, 4)
    assert need > 0
    def attend(ws=P, n=need, **kw):
        a = attention(**kw)  # (alive during the call)
        return LIB.rps_tree_attention_fwd(at(a), at(kv), ws, n, None)

    for kw in (dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 2), dict(layer=2), dict(layer=-1), dict(n_q=0),
               dict(n_heads=6), dict(n_heads=0), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(q_seq_stride=4), dict(q_token_stride=0), dict(q_head_stride=-8), dict(out_seq_stride=1),
               dict(out_token_stride=-512), dict(out_head_stride=0), dict(ws=None), dict(ws=P + 8), dict(n=need - 1)):
        assert attend(**kw) == BAD, kw
    for kw in (dict(n_q=1025), dict(n_heads=4 * 129)):
        assert attend(**kw) == BEYOND, kw
    assert LIB.rps_tree_attention_fwd(None, at(kv), P, need, None) == BAD


def test_turns_are_the_fraction_of_a_turn():
    for f in (1.0, 0.5, 1e-3, 500000.0 ** -0.9, 2.0 * math.pi, 100.0, -0.25, 0.0):
        got = Fraction(rps._lib.rps_rope_turns(f), 1 << 64)
        exact = Fraction(f) / (2 * Fraction(math.pi)) % 1  # pi to 53 bits: what the double division sees
        off = abs(got - exact)
        assert min(off, 1 - off) <= Fraction(abs(f) + 1e-3) * Fraction(1, 1 << 52), f
    assert all(rps._lib.rps_rope_turns(f) == 0 for f in (float("inf"), float("-inf"), float("nan")))


def test_frequencies_of_scaled_contexts():
    plain, one = rps.rope_inv_freq(64, 10000.0)
    assert one == 1.0 and len(plain) == 32 and plain[0] == 1.0 and math.isclose(plain[16], 0.01)
    assert rps.rope_inv_freq(64, 10000.0, linear=4.0)[0] == [f / 4.0 for f in plain]
    parts, amplitude = rps.rope_inv_freq(64, 10000.0, parts=(8.0, 4096, 32.0, 1.0))
    assert math.isclose(amplitude, 0.1 * math.log(8.0) + 1.0)
    for f, g in zip(plain, parts):
        turns = 4096 * f / (2 * math.pi)
        assert g == f if turns >= 32 else math.isclose(g, f / 8) if turns <= 1 else f / 8 < g < f
    for bad in ((0.5, 4096, 32.0, 1.0), (8.0, 0, 32.0, 1.0), (8.0, 4096, 1.0, 1.0)):
        with pytest.raises(ValueError):
            rps.rope_inv_freq(64, parts=bad)


def test_oracle_of_drafted_tokens():
    sees, depth, bad = drafts.masks([-1, 0, 0, 1, -1], 5)
    assert not bad and depth.tolist() == [0, 1, 1, 2, 0]
    assert [np.flatnonzero(r).tolist() for r in sees] == [[0], [0, 1], [0, 2], [0, 1, 3], [4]]
    assert drafts.masks([-1, 1, 7], 3)[2] and drafts.words(np.tril(np.ones((40, 40), bool)))[39].tolist() == [-1, 255]
    # a kept path in order, and what it leaves alone
    k = np.arange(2 * 16, dtype=np.float64).reshape(1, 2, 1, 16, 1)
    c = Cache([1, 1], [[0, 1]], [18], 16, k.copy(), k.copy())
    assert drafts.keep_path(c, [[1, 2, 5]], [3], 6).tolist() == [15]
    assert c.k[0, 0, 0, 12:, 0].tolist() == [13, 14, 17, 15] and c.err == 0
    assert drafts.keep_path(c, [[2, 2]], [2], 6).tolist() == [18] and c.err == drafts.DEVERR_ROW_INDEX
    # a rotation keeps a pair's length, and turns by the position
    y, _ = drafts.rotate([3.0, 4.0], None, 0.0, [0.5], True, 1.0, math.pi)
    assert np.allclose(y, [-4.0, 3.0])
