"""Attention over the paged K/V cache (rps_prefix_attention_fwd) against the oracle
(oracle/kvcache.py, one query at a time in fp64).

Tolerance, from the arithmetic: a probability is rounded to the cache's type before
it weights the values, by at most half a step e (bf16 2^-8, fp16 2^-11), and the
output is rounded by as much, so |out - ref| <= e (sum_k p_k |v_k| + |ref|) up to
fp32 terms. fp16 probabilities below 2^-14 are rounded by at most 2^-25 each, against
a sum of at least 2^-8 (the reference lags the largest score by at most 8 units of
base 2): 2^-17 max |v| for n keys of which each weighs less than that, bounded by
n 2^-25 max |v| / sum; with the sums here (above 1) n 2^-25 max |v|. The fp32 terms:
a score of 128 products with |q||k| below 2^9 is off by at most 2^-24 * 128 * 2^9 / 64
in relative weight, 2^-14 at the worst; allowed as 2^-12 of the weighted |v|.
lse: fp32 scores and sums, 2^-12 absolute by the same bound, and log and exp of fp32.
"""
import numpy as np
import pytest
import torch

from oracle import kvcache as ok
from paper_2608_11742_gb300 import rps, synth

pytestmark = pytest.mark.gpu

D = 128
EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def rounded(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dtype)


class Case:
    """lens [n_req][n_branch], shared [n_req] tokens: pages below it are the same ids for the request's sequences.
    Everything that no query may see is NaN."""

    def __init__(self, seed, lens, shared, n_q, H, Hk, ps, dtype=torch.bfloat16, causal=False, layers=1, layer=0,
                 tokens_first=False, growth=0.0, spare=3, scale=D ** -0.5, wide=False):
        rng = np.random.default_rng(seed)
        lens = np.array(lens)
        self.lens, self.shared, self.n_q, self.H, self.causal, self.layer = lens, shared, n_q, H, causal, layer
        self.scale, self.dtype, self.ps = scale, dtype, ps
        n_req, nb = lens.shape
        pages = lambda n: 0 if n <= 0 else -(-int(n) // ps)
        width = max(1, max(pages(n) for n in lens.ravel())) + 1
        if wide:  # a table far wider than the sequences need: more CTAs than key tiles
            width = max(width, -(-2560 * 128 // (ps * n_req * Hk * -(-nb * n_q // (128 // (H // Hk))))) + 16)
        table, count = np.full((n_req, nb, width), -1), 0
        for r in range(n_req):
            common = max(0, shared[r]) // ps if shared is not None else 0
            for i in range(common):
                holders = [b for b in range(nb) if pages(lens[r, b]) > i]
                if holders:
                    table[r, holders, i] = count
                    count += 1
            for b in range(nb):
                for i in range(min(common, pages(lens[r, b])), pages(lens[r, b])):
                    table[r, b, i] = count
                    count += 1
        n_pages = count + spare
        place = rng.permutation(n_pages)
        table = np.where(table >= 0, place[table], -1)
        # data: NaN everywhere but at the tokens some sequence holds
        k = torch.full((layers, n_pages, Hk, ps, D), float("nan"), dtype=dtype)
        v = k.clone()
        for r in range(n_req):
            for b in range(nb):
                for i in range(pages(lens[r, b])):
                    m = min(ps, lens[r, b] - i * ps)
                    p = table[r, b, i]
                    for l in range(layers):
                        if bool(torch.isnan(k[l, p, :, :m].float()).any()):
                            x = rng.standard_normal((2, Hk, m, D))
                            if growth:
                                x[0] *= 1.0 + growth * ((i * ps + np.arange(m)) // 128)[None, :, None]
                            k[l, p, :, :m], v[l, p, :, :m] = rounded(x[0], dtype), rounded(x[1], dtype)
        self.q = rounded(2.0 * rng.standard_normal((n_req, nb, n_q, H, D)), dtype)
        self.k, self.v, self.table = k, v, table
        dk, dv = k.cuda(), v.cuda()
        if tokens_first:
            dk, dv = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (dk, dv))
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
        ref = np.bincount(table[table >= 0].ravel(), minlength=n_pages)
        self.kv = rps.KvCacheBuf(dk, dv, i32(ref), i32(table), i32(lens))
        self.d_shared = None if shared is None else i32(shared)
        self.dq = self.q.cuda()
        self.ws = torch.full((rps.rps_prefix_attention_workspace_bytes(self.kv, n_q, H),), 255, dtype=torch.uint8,
                             device="cuda")

    def run(self, out=None, lse=True, stream=None):
        n_req, nb, n_q, H, _ = self.q.shape
        out = torch.full(self.q.shape, 7.0, dtype=self.dtype, device="cuda") if out is None else out
        z = torch.full((n_req, nb, n_q, H), 7.0, dtype=torch.float32, device="cuda") if lse else None
        rps.rps_prefix_attention_fwd(self.dq, self.kv, self.layer, out, self.ws, self.d_shared, self.scale, self.causal,
                                     z, stream)
        return out, z

    def reference(self):
        n = self.lens.size
        pages = [np.nan_to_num(x.double().numpy()) for x in (self.k, self.v)]
        c = ok.Cache(np.ones(self.k.shape[1]), self.table.reshape(n, -1), self.lens.reshape(n), self.ps, *pages)
        q = self.q.double().numpy().reshape(n, *self.q.shape[2:])
        scale = float(np.float32(self.scale))
        return [x.reshape(*self.lens.shape, *x.shape[1:]) for x in ok.prefix_attention(q, c, self.layer, scale, self.causal)]

    def check(self, out, lse, where=None, detail=0):
        status, bits = rps.rps_poll_device_status()
        assert bits == detail, hex(bits)
        ref, mag, z = self.reference()
        g = out.double().cpu().numpy()
        absent = np.isnan(ref)
        keep = np.ones(ref.shape[:2], bool) if where is None else where
        assert (g[absent] == 7.0).all(), "rows of absent sequences were written"
        e = EPS[self.dtype]
        tiny = 2.0 ** -25 * max(0, self.lens.max()) * 5.0 if self.dtype == torch.float16 else 0.0
        tol = e * (mag + np.abs(ref)) + 2.0 ** -12 * mag + tiny + 1e-6
        bad = ~(np.abs(g - ref) <= tol) & ~absent & keep[:, :, None, None, None]
        assert not bad.any(), (f"{bad.sum()} of {bad.size} outputs out of tolerance, worst "
                               f"{np.nanmax(np.abs(g - ref)[bad]):.3e} at {np.argwhere(bad)[:3].tolist()}")
        if lse is not None:
            h = lse.double().cpu().numpy()
            here = ~np.isnan(z) & keep[:, :, None, None]
            assert (h[np.isnan(z)] == 7.0).all()
            with np.errstate(invalid="ignore"):
                fine = (h == z) | (np.abs(h - z) <= 2.0 ** -12 + 2.0 ** -20 * np.abs(z))
            assert fine[here].all(), f"lse differs by {np.abs(h - z)[here & ~fine].max()}"
        return g


CASES = {
    # one sequence, one token of context: everything is one key
    "one key": dict(lens=[[1]], shared=None, n_q=1, H=1, Hk=1, ps=16),
    "whole tiles, no sharing": dict(lens=[[256]], shared=None, n_q=128, H=1, Hk=1, ps=64),
    "ragged tail": dict(lens=[[133]], shared=None, n_q=3, H=2, Hk=2, ps=16),
    "lengths around a page and a tile": dict(lens=[[15, 16, 17], [127, 128, 129]], shared=None, n_q=1, H=2, Hk=1, ps=16),
    "branches on a shared context": dict(lens=[[168] * 9], shared=[136], n_q=32, H=2, Hk=2, ps=16),
    "shared and own, ragged": dict(lens=[[300, 289, 256, 331], [64, 40, 70, 33]], shared=[256, 32], n_q=5, H=4, Hk=2, ps=32),
    "seven heads a group": dict(lens=[[500, 470, 480]], shared=[448], n_q=9, H=14, Hk=2, ps=64),
    "more sequences than a tile": dict(lens=[[70 + 3 * (i % 7) for i in range(150)]], shared=[64], n_q=1, H=1, Hk=1, ps=16),
    "absent and empty": dict(lens=[[40, -1, 0, 33, -1], [-1] * 5, [0] * 5, [-1, -1, 20, 17, -1]], shared=[32, 0, 16, 16],
                             n_q=4, H=2, Hk=1, ps=16),
    "pages of 256": dict(lens=[[700, 513, 512], [256, 255, 300]], shared=[512, 256], n_q=2, H=4, Hk=2, ps=256),
    "pages of 128": dict(lens=[[700, 513, 640], [256, 255, 300]], shared=[512, 128], n_q=2, H=4, Hk=2, ps=128),
    "long, split over many CTAs": dict(lens=[[9000, 8990]], shared=[8980], n_q=1, H=3, Hk=1, ps=64),
    "long own parts": dict(lens=[[2000, 1500, 16, 900]], shared=[16], n_q=2, H=2, Hk=1, ps=16),
    "many small row tiles": dict(lens=[[20 + (i * 7 + j) % 30 for j in range(3)] for i in range(60)], shared=[16] * 60,
                                 n_q=2, H=8, Hk=8, ps=16),
    "group of 128": dict(lens=[[77, 90]], shared=[64], n_q=2, H=128, Hk=1, ps=16),
    "two halves and one, many heads": dict(lens=[[150, 140, 161, 133, 155], [260, 241, 250, 255, 245]], shared=[128, 240],
                                           n_q=32, H=6, Hk=6, ps=16),
    "sequences across the halves": dict(lens=[[400, 390, 380]], shared=[352], n_q=100, H=2, Hk=1, ps=32),
    "shared length beyond the sequences": dict(lens=[[100, 60, 250]], shared=[1000], n_q=3, H=2, Hk=2, ps=32),
}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_parity(name, wide, causal):
    c = Case(21, causal=causal, dtype=torch.float16 if len(name) % 2 else torch.bfloat16, wide=wide, **CASES[name])
    c.check(*c.run())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_types_layers_and_layouts(dtype, tokens_first):
    c = Case(22, [[90, 77], [64, 130]], [64, 48], 3, 4, 2, 16, dtype, True, layers=3, layer=1, tokens_first=tokens_first)
    c.check(*c.run())
    # q and out as slices of wider rows, heads outermost
    n_req, nb, n_q, H, _ = c.q.shape
    wide = torch.full((n_req, H, nb * n_q, 3 * D), 7.0, dtype=dtype, device="cuda")
    view = lambda x, at: x[..., at:at + D].view(n_req, H, nb, n_q, D).permute(0, 2, 3, 1, 4)
    view(wide, 0).copy_(c.q)
    c.dq = view(wide, 0)
    out = view(wide, D)
    c.check(*c.run(out))
    assert bool((wide[..., 2 * D:] == 7.0).all()) and torch.equal(view(wide, 0).cpu(), c.q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ps", [16, 64, 256])
def test_pages_at_odd_strides(ps, dtype):
    """Pages whose distance is no multiple of eight tokens', and one that is, with tokens wider than they are read;
    a page id outside the cache among them."""
    for pad, extra in ((1, 0), (0, 8), (3, 8)):
        c = Case(24, [[90, 77, 300], [64, 513, 1]], [64, 0], 3, 6, 3, ps, dtype, True)
        for name in ("k", "v"):
            t = getattr(c.kv, name)
            layers, pages, heads = t.shape[:3]
            to = torch.full((layers, pages, heads * ps + pad, D + extra), float("nan"), dtype=dtype, device="cuda")
            view = to[:, :, :heads * ps].view(layers, pages, heads, ps, D + extra)[..., :D] if pad == 0 else to.as_strided(
                t.shape, (to.stride(0), to.stride(1), ps * (D + extra), D + extra, 1))
            view.copy_(t)
            setattr(c.kv, name, view)
        c.check(*c.run())
        whole = c.run()
        c.kv.table[1, 1, 0] = c.kv.k.shape[1] + 5
        out, lse = c.run()[:2]
        assert rps.rps_poll_device_status() == (rps.RPS_ERR_DEVICE, rps.DEVERR_PAGE)
        assert bool(torch.isnan(out[1, 1]).all()) and bool(torch.isnan(lse[1, 1]).all())
        keep = torch.ones((2, 3), dtype=torch.bool)
        keep[1, 1] = False
        assert torch.equal(out[keep], whole[0][keep])


@pytest.mark.parametrize("causal", [False, True])
def test_more_row_tiles_than_a_block_has_threads(causal):
    """700 requests of two sequences, some absent: the plan goes through two blocks of row tiles, lengths and key tiles
    are read again instead of kept."""
    rng = np.random.default_rng(27)
    lens = rng.integers(1, 60, (700, 2))
    lens[rng.random((700, 2)) < 0.15] = -1
    lens[300:310] = -1
    c = Case(27, lens, [int(x) for x in rng.integers(0, 40, 700)], 1, 2, 2, 16, causal=causal)
    c.check(*c.run())


@pytest.mark.parametrize("group,n_q", [(2, 64), (128, 1)])
def test_many_row_tiles_of_a_request(group, n_q):
    """70 row tiles of a head: the range's begin is found in more than a warp's width of them."""
    nb = 70
    c = Case(28, [[200 + 5 * (i % 9) for i in range(nb)], [66] * nb], [192, 64], n_q, 2 * group, 2, 32, causal=True)
    c.check(*c.run())


def test_causal_rows_longer_than_the_sequence():
    """n_q beyond a sequence's length: the first queries see nothing, their rows are zero."""
    c = Case(23, [[5, 130, 20]], [0], 24, 2, 1, 16, causal=True)
    out, lse = c.run()
    c.check(out, lse)
    assert bool((out[0, 0, :19] == 0).all()) and bool(torch.isinf(lse[0, 0, :19]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", [0.3, 3.0, 1e-4])
def test_scores_that_grow_are_rescaled(dtype, scale):
    """Scores far above and below the reference that a row starts with."""
    c = Case(24, [[700, 690]], [640], 4, 2, 1, 64, dtype, growth=1.0, scale=scale)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scores_that_are_all_far_below_zero(dtype):
    """Every score about -1400 to -200 in base 2: a weight of 2^score would vanish."""
    c = Case(31, [[300, 290]], [256], 4, 2, 1, 64, dtype)
    c.q[..., 0], c.q[..., 1:] = 16.0, c.q[..., 1:] * 0.25
    for name in ("k",):
        x = getattr(c, name)
        x[..., 0] = torch.where(torch.isnan(x[..., 0]), x[..., 0], -20.0 - 2.0 * torch.rand(x[..., 0].shape).to(dtype))
    c.scale = 1.0
    c.dq, c.kv.k = c.q.cuda(), c.k.cuda()
    c.check(*c.run())


def test_scores_without_weight():
    """Keys whose scores are -inf for every query take no weight; a row with no others is zero."""
    c = Case(25, [[150, 140], [40, 40]], [128, 32], 2, 2, 1, 16)
    c.q[..., 0] = 1.0
    c.k[:, :, :, :, 0] = torch.where(torch.isnan(c.k[:, :, :, :, 0]), float("nan"), 0.0)
    for i in range(8):
        c.k[0, c.table[0, 0, i], :, :, 0] = -float("inf")  # the shared pages of the first request
    for b in range(2):
        for i in range(3):
            c.k[0, c.table[1, b, i], :, :, 0] = -float("inf")  # all of the second
    c.dq, c.kv.k = c.q.cuda(), c.k.cuda()
    out, lse = c.run()
    ref_k = c.k.clone()
    c.k = torch.where(torch.isinf(c.k), torch.tensor(-3e4, dtype=c.k.dtype), c.k)
    ref, mag, z = c.reference()
    g, h = out.double().cpu().numpy(), lse.cpu().numpy()
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert (np.abs(g - ref)[0] <= EPS[c.dtype] * (mag + np.abs(ref))[0] + 2.0 ** -12 * mag[0] + 1e-6).all()
    assert (g[1] == 0).all() and np.isneginf(h[1]).all() and (np.abs(h - z)[0] <= 2.0 ** -11).all()


def test_bad_pages_give_nan_to_the_rows_that_see_them():
    c = Case(26, [[200, 190, 180], [100, 90, 80]], [160, 64], 2, 2, 2, 16)
    c.kv.table[0, 1, 11] = c.k.shape[1]  # an own page of one sequence
    c.kv.table[1, 0, 2] = -3             # a shared page, in the row that is read for all
    out, lse = c.run()
    where = np.array([[True, False, True], [False] * 3])
    c.check(out, lse, where, detail=rps.DEVERR_PAGE)
    assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isnan(out[1]).all()) and bool(torch.isnan(lse[1]).all())


def test_a_sequence_does_not_reach_another():
    """inf and NaN in one sequence's own keys and values change no bit of the others."""
    kw = dict(lens=[[200, 177, 190, 181]], shared=[160], n_q=3, H=2, Hk=1, ps=16)
    a, b = Case(27, **kw), Case(27, **kw)
    for i in (10, 11):
        b.k[0, b.table[0, 1, i]] = float("nan")
        b.v[0, b.table[0, 1, i]] = float("inf")
    b.kv.k, b.kv.v = b.k.cuda(), b.v.cuda()
    x, y = a.run()[0], b.run()[0]
    others = [0, 2, 3]
    assert torch.equal(x[:, others], y[:, others])
    assert bool(torch.isnan(y[:, 1]).all())


def test_repeats_bit_for_bit_on_a_side_stream_and_from_a_graph():
    c = Case(28, [[700, 650, 666], [128, 90, -1]], [640, 64], 8, 4, 2, 16)
    first = c.run()[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.full_like(first, 7.0)
    with torch.cuda.stream(side):
        c.run(out, stream=side)
    side.synchronize()
    assert torch.equal(out, first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.run(out, lse=False)
    for _ in range(3):
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
    # the graph reads the lengths it finds
    c.lens = np.array([[650, -1, 666], [100, 90, 70]])
    c.kv.table[1, 2, :8] = c.kv.table[1, 0, :8]
    c.table[1, 2, :8] = c.table[1, 0, :8]
    c.kv.length.copy_(torch.from_numpy(c.lens))
    out.fill_(7.0)
    g.replay()
    c.check(out, None)


def test_wait_timeout_is_reported_and_the_next_launch_works():
    c = Case(29, [[300, 290]], [256], 4, 2, 1, 16)
    torch.cuda.synchronize()
    rps.rps_debug_set_ring_wait_ns(0)
    try:
        c.run()
        status, detail = rps.rps_poll_device_status()
    finally:
        rps.rps_debug_set_ring_wait_ns(2 ** 64 - 1)
    assert status == rps.RPS_ERR_DEVICE and detail & rps.DEVERR_TIMEOUT, hex(detail)
    c.check(*c.run())


def test_refusals_of_the_binding():
    c = Case(30, [[40, 33]], [32], 2, 4, 2, 16)
    args = lambda **kw: {**dict(q=c.dq, kv=c.kv, layer=0, out=torch.empty_like(c.dq), ws=c.ws, shared_len=c.d_shared,
                                scale=0.1), **kw}
    for kw, err in ((dict(q=c.dq.float()), TypeError), (dict(out=torch.empty_like(c.dq, dtype=torch.float16)), TypeError),
                    (dict(q=c.dq[:, :1]), ValueError), (dict(out=c.dq[..., :64]), ValueError),
                    (dict(q=c.q), ValueError), (dict(shared_len=c.d_shared.long()), ValueError),
                    (dict(lse=torch.empty(3, device="cuda")), ValueError), (dict(ws=c.ws[:-1]), rps.RPSError),
                    (dict(layer=1), rps.RPSError), (dict(scale=0.0), rps.RPSError),
                    (dict(scale=float("inf")), rps.RPSError)):
        with pytest.raises(err):
            rps.rps_prefix_attention_fwd(**args(**kw))
    three = torch.zeros((1, 2, 2, 3, D), dtype=c.dtype, device="cuda")
    with pytest.raises(rps.RPSError):  # heads that are no multiple of the cache's
        rps.rps_prefix_attention_fwd(**args(q=three, out=torch.empty_like(three)))
