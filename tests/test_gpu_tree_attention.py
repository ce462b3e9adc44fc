"""Attention of drafted tokens over the paged K/V cache (rps_tree_attention_fwd) against the
oracle (oracle/drafts.py, one query at a time in fp64).

Tolerance: as for the attention of branches (test_gpu_prefix_attention.py), whose arithmetic
is the same: a probability and the output rounded to the cache's type, half a step each, and
2^-12 of the weighted |v| for the fp32 scores.
"""
import numpy as np
import pytest
import torch

from oracle import drafts
from oracle import kvcache as ok
from paper_2608_11742_gb300 import rps
from test_gpu_prefix_attention import Case, D

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


class Tree(Case):
    """lens [n_req][n_branch] with the drafted tokens; count: drafted tokens of each sequence (None: n_q); sees: "tree",
    "chain" (no mask), "none" (no bit set), "all", or truth values [n_seq][n_q][n_q]."""

    def __init__(self, seed, lens, n_q, H, Hk, ps, count=None, sees="tree", **kw):
        kw.pop("shared", None)
        super().__init__(seed, lens, None, n_q, H, Hk, ps, **kw)
        n = self.lens.size
        rng = np.random.default_rng(seed + 1000)
        self.count = None if count is None else np.array(count)
        if isinstance(sees, str):
            full = {"chain": None, "none": np.zeros((n, n_q, n_q), bool), "all": np.ones((n, n_q, n_q), bool)}.get(sees, 0)
            if sees == "tree":
                full = np.stack([drafts.masks([int(rng.integers(-1, i)) if i else -1 for i in range(n_q)], n_q)[0] for _ in range(n)])
            sees = full
        self.sees = sees
        self.mask = None if sees is None else i32(np.stack([drafts.words(x) for x in sees]))
        self.d_count = None if count is None else i32(count)
        self.ws = torch.full((rps.rps_tree_attention_workspace_bytes(self.kv, n_q, H),), 255, dtype=torch.uint8, device="cuda")

    def run(self, out=None, lse=True, stream=None):
        n_req, nb, n_q, H, _ = self.q.shape
        out = torch.full(self.q.shape, 7.0, dtype=self.dtype, device="cuda") if out is None else out
        z = torch.full((n_req, nb, n_q, H), 7.0, dtype=torch.float32, device="cuda") if lse else None
        rps.rps_tree_attention_fwd(self.dq, self.kv, self.layer, out, self.ws, self.mask, self.scale, self.d_count, z, stream)
        return out, z

    def reference(self):
        n = self.lens.size
        pages = [np.nan_to_num(x.double().numpy()) for x in (self.k, self.v)]
        c = ok.Cache(np.ones(self.k.shape[1]), self.table.reshape(n, -1), self.lens.reshape(n), self.ps, *pages)
        q = self.q.double().numpy().reshape(n, *self.q.shape[2:])
        got = drafts.tree_attention(q, c, self.layer, float(np.float32(self.scale)), self.count, self.sees)
        return [x.reshape(*self.lens.shape, *x.shape[1:]) for x in got]


CASES = {
    "one key": dict(lens=[[1]], n_q=1, H=1, Hk=1, ps=16),
    "single tokens": dict(lens=[[1], [15], [16], [17], [127], [128], [129], [700], [0], [-1]], n_q=1, H=14, Hk=2, ps=16),
    "a small tree": dict(lens=[[133]], n_q=9, H=2, Hk=2, ps=16),
    "the tree alone": dict(lens=[[40], [40]], n_q=40, H=4, Hk=2, ps=16),
    "trees across tiles": dict(lens=[[140], [128 + 33], [256 + 1], [300]], n_q=33, H=2, Hk=1, ps=32),
    "pairs of row tiles": dict(lens=[[300], [129], [90]], n_q=64, H=4, Hk=1, ps=64),
    "pairs, the last alone": dict(lens=[[500], [333]], n_q=70, H=7, Hk=1, ps=16),
    "pairs and fewer tokens": dict(lens=[[300], [290], [280], [270], [100]], n_q=64, H=4, Hk=1, ps=64, count=[64, 31, 1, 33, 0]),
    "ragged": dict(lens=[[60, 33, -1], [20, 90, 8]], n_q=12, H=6, Hk=3, ps=16, count=[12, 1, 5, 0, 7, 99]),
    "longer than the sequence": dict(lens=[[5], [12], [1]], n_q=12, H=2, Hk=1, ps=16),
    "groups of 128": dict(lens=[[77], [20]], n_q=3, H=128, Hk=1, ps=16),
    "groups of 65": dict(lens=[[77], [200]], n_q=3, H=130, Hk=2, ps=16),
    "long, over many CTAs": dict(lens=[[9000], [4001]], n_q=4, H=3, Hk=1, ps=64),
    "long pairs": dict(lens=[[5000]], n_q=40, H=8, Hk=2, ps=128),
    "pages of 256": dict(lens=[[700], [513], [256]], n_q=5, H=4, Hk=2, ps=256),
    "many short sequences": dict(lens=[[10 + 3 * (i % 29)] for i in range(170)], n_q=2, H=4, Hk=2, ps=16),
}


@pytest.mark.parametrize("sees", ["tree", "chain"])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_parity(name, wide, sees):
    c = Tree(21, sees=sees, dtype=torch.float16 if len(name) % 2 else torch.bfloat16, wide=wide, **CASES[name])
    c.check(*c.run())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_types_layers_and_layouts(dtype, tokens_first):
    c = Tree(22, [[90, 77], [64, 130]], 11, 4, 2, 16, dtype=dtype, layers=3, layer=1, tokens_first=tokens_first)
    c.check(*c.run())
    # q and out as slices of wider rows, heads outermost
    n_req, nb, n_q, H, _ = c.q.shape
    wide = torch.full((n_req * nb, H, n_q, 3 * D), 7.0, dtype=dtype, device="cuda")
    view = lambda x, at: x[..., at:at + D].view(n_req, nb, H, n_q, D).permute(0, 1, 3, 2, 4)
    view(wide, 0).copy_(c.q)
    c.dq = view(wide, 0)
    c.check(*c.run(view(wide, D)))
    assert bool((wide[..., 2 * D:] == 7.0).all()) and torch.equal(view(wide, 0).cpu(), c.q)


@pytest.mark.parametrize("n_q", [5, 40])
def test_rows_off_the_sectors(n_q):
    """Queries and outputs whose rows begin 16 bytes off the 32-byte bounds: bit for bit as others; units whole and cut."""
    c = Tree(49, [[90], [5000]], n_q, 8, 2, 16)
    first, z = c.run()
    wide = torch.full((2, 1, n_q, 8, D + 8), 7.0, dtype=c.dtype, device="cuda")
    wide[..., 8:] = c.dq
    c.dq = wide[..., 8:]
    to = torch.full_like(wide, 7.0)
    out, lse = c.run(to[..., 8:])
    assert torch.equal(out, first) and torch.equal(lse, z) and bool((to[..., :8] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ps", [16, 256])
def test_pages_at_odd_strides(ps, dtype):
    """Pages whose distance is no multiple of eight tokens', and tokens wider than they are read."""
    for pad, extra in ((1, 0), (0, 8), (3, 8)):
        c = Tree(24, [[90, 77, 300], [64, 513, 8]], 7, 6, 3, ps, dtype=dtype)
        for name in ("k", "v"):
            t = getattr(c.kv, name)
            layers, pages, heads = t.shape[:3]
            to = torch.full((layers, pages, heads * ps + pad, D + extra), float("nan"), dtype=dtype, device="cuda")
            view = to.as_strided(t.shape, (to.stride(0), to.stride(1), ps * (D + extra), D + extra, 1))
            view.copy_(t)
            setattr(c.kv, name, view)
        c.check(*c.run())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_masks_that_leave_nothing(dtype):
    """No bit set: the context alone, and where there is none, zeros."""
    c = Tree(25, [[30], [200], [9]], 9, 4, 2, 16, sees="none", dtype=dtype)
    out, lse = c.run()
    c.check(out, lse)
    assert bool((out[2] == 0).all()) and bool(torch.isneginf(lse[2]).all())
    c = Tree(26, [[140]], 40, 8, 2, 16, sees="all", dtype=dtype)
    c.check(*c.run())


def test_bits_past_a_sequences_tokens_are_not_looked_at():
    a = Tree(27, [[60], [33]], 40, 2, 1, 16, count=[7, 33])
    first = a.run()[0].clone()
    a.mask[0] |= i32([-1 << 7, -1])  # (tokens 7.. of the first sequence)
    a.mask[1] |= i32([0, -2])
    assert torch.equal(a.run()[0], first)


def test_keys_that_a_row_does_not_see_may_hold_anything():
    """NaN and inf in a drafted token's key change no bit of the rows that do not see it."""
    sees = np.zeros((1, 20, 20), bool)
    sees[0, np.arange(20), np.arange(20)] = True
    a, b = (Tree(28, [[150]], 20, 4, 2, 16, sees=sees) for _ in range(2))
    for t, value in ((133, float("nan")), (140, float("inf")), (141, -float("inf"))):
        b.k[0, b.table[0, 0, t // 16], :, t % 16] = value
    b.kv.k = b.k.cuda()
    x, y = a.run()[0], b.run()[0]
    rest = [i for i in range(20) if i not in (3, 10, 11)]
    assert torch.equal(x[0, 0, rest], y[0, 0, rest])
    assert bool(torch.isnan(y[0, 0, 3]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", [0.3, 3.0, 1e-4])
@pytest.mark.parametrize("n_q", [4, 40])
def test_scores_that_grow_are_rescaled(n_q, scale, dtype):
    c = Tree(29, [[1500], [690]], n_q, 8, 1, 64, dtype=dtype, growth=1.0, scale=scale)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scores_that_are_all_far_below_zero(dtype):
    c = Tree(31, [[300], [290]], 4, 2, 1, 64, dtype=dtype)
    c.q[..., 0], c.q[..., 1:] = 16.0, c.q[..., 1:] * 0.25
    x = c.k
    x[..., 0] = torch.where(torch.isnan(x[..., 0]), x[..., 0], -20.0 - 2.0 * torch.rand(x[..., 0].shape).to(dtype))
    c.scale = 1.0
    c.dq, c.kv.k = c.q.cuda(), c.k.cuda()
    c.check(*c.run())


def test_scores_without_weight():
    """Keys whose scores are -inf take no weight; a row with no others is zero."""
    c = Tree(32, [[150], [40]], 2, 2, 1, 16, sees="chain")
    c.q[..., 0] = 1.0
    c.k[..., 0] = torch.where(torch.isnan(c.k[..., 0]), float("nan"), 0.0)
    for i in range(5):
        c.k[0, c.table[0, 0, i], :, :, 0] = -float("inf")
    for i in range(3):
        c.k[0, c.table[1, 0, i], :, :, 0] = -float("inf")
    c.dq, c.kv.k = c.q.cuda(), c.k.cuda()
    out, lse = c.run()
    c.k = torch.where(torch.isinf(c.k), torch.tensor(-3e4, dtype=c.k.dtype), c.k)
    ref, mag, z = c.reference()
    g, h = out.double().cpu().numpy(), lse.cpu().numpy()
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert (np.abs(g - ref)[0] <= 2.0 ** -8 * (mag + np.abs(ref))[0] + 2.0 ** -12 * mag[0] + 1e-6).all()
    assert (g[1] == 0).all() and np.isneginf(h[1]).all() and (np.abs(h - z)[0] <= 2.0 ** -11).all()


@pytest.mark.parametrize("n_q", [3, 70])
def test_bad_pages_give_nan_to_the_rows_that_see_them(n_q):
    c = Tree(33, [[200, 190], [100, 90]], n_q, 4, 2, 16, sees="chain")
    whole = c.run()[0].clone()
    c.kv.table[0, 1, 2] = c.k.shape[1]
    c.kv.table[1, 0, 6] = -3  # tokens 96.. of 100: drafted ones
    out, lse = c.run()
    assert rps.rps_poll_device_status() == (rps.RPS_ERR_DEVICE, rps.DEVERR_PAGE)
    assert torch.equal(out[0, 0], whole[0, 0]) and torch.equal(out[1, 1], whole[1, 1])
    assert bool(torch.isnan(out[0, 1]).all()) == (190 - n_q >= 32) and bool(torch.isnan(out[0, 1, -1]).all())
    first = n_q - 4  # the query that is token 96
    assert bool(torch.isnan(out[1, 0, max(0, first):]).all())
    if first > 0:
        assert torch.equal(out[1, 0, :first], whole[1, 0, :first])


@pytest.mark.parametrize("n_q", [3, 70])
@pytest.mark.parametrize("pad", [0, 1])
def test_page_ids_far_outside_the_cache(n_q, pad):
    """Ids whose low bits are those of a page of the cache are outside it, too; pages in groups of eight tokens, and one by one."""
    for bad in (-2 ** 31, -2 ** 31 + 1, -1, 2 ** 31 - 1, 2 ** 30):
        c = Tree(50, [[200, 190], [100, 90]], n_q, 4, 2, 16, sees="chain")
        if pad:
            for name in ("k", "v"):
                t = getattr(c.kv, name)
                to = torch.full((*t.shape[:2], t.shape[2] * 16 + pad, D), float("nan"), dtype=c.dtype, device="cuda")
                view = to.as_strided(t.shape, (to.stride(0), to.stride(1), 16 * D, D, 1))
                view.copy_(t)
                setattr(c.kv, name, view)
        whole = c.run()[0].clone()
        c.kv.table[0, 1, 2] = bad  # tokens 32.. of 190
        c.kv.table[1, 0, 6] = bad  # tokens 96.. of 100: drafted ones
        out, lse = c.run()
        assert rps.rps_poll_device_status() == (rps.RPS_ERR_DEVICE, rps.DEVERR_PAGE)
        assert torch.equal(out[0, 0], whole[0, 0]) and torch.equal(out[1, 1], whole[1, 1])
        assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isnan(lse[0, 1]).all())
        first = max(0, n_q - 4)  # the query that is token 96
        assert bool(torch.isnan(out[1, 0, first:]).all()) and torch.equal(out[1, 0, :first], whole[1, 0, :first])


def test_lengths_beyond_the_table():
    c = Tree(34, [[100], [64]], 4, 2, 1, 16)
    width = c.table.shape[2]
    c.kv.length[1] = 100000
    c.kv.table[1, 0] = c.kv.table[0, 0]
    c.kv.table[1, 0, -1] = c.kv.table[0, 0, 0]
    out, _ = c.run()
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK and width * 16 > 100
    assert bool(torch.isfinite(out[0]).all())


@pytest.mark.parametrize("n_seq", [383, 384, 385, 639, 640, 641, 1000])
def test_more_sequences_than_a_block_has_threads(n_seq):
    rng = np.random.default_rng(35)
    lens = rng.integers(1, 40, (n_seq, 1))
    lens[rng.random((n_seq, 1)) < 0.1] = -1
    lens[300:330] = -1
    c = Tree(35, lens, 2, 2, 2, 16, sees="chain")
    c.check(*c.run())


@pytest.mark.parametrize("sees", ["tree", "chain"])
@pytest.mark.parametrize("n_q", [4, 70])
def test_lengths_beyond_the_table_count_as_its_capacity(n_q, sees):
    """All rows, and the positions of the drafted tokens among them: bit for bit as a full table, in single row tiles and pairs."""
    c = Tree(52, [[100], [320], [256], [320]], n_q, 4, 1, 16, sees=sees, count=[n_q, n_q - 1, n_q, 2])
    width = c.table.shape[2] - 1  # (the case's own spare column)
    assert width == 20
    c.kv = rps.KvCacheBuf(c.kv.k, c.kv.v, c.kv.page_ref, c.kv.table[..., :width].contiguous(), c.kv.length)
    first, z = c.run()
    c.check(first, z)
    for beyond in (321, 1000, 2 ** 31 - 1):
        c.kv.length[1], c.kv.length[3] = beyond, beyond
        out, lse = c.run()
        c.check(out, lse)
        assert torch.equal(out, first) and torch.equal(lse, z)


@pytest.mark.parametrize("n_seq", [1023, 1024, 1025, 1500, 5000])
@pytest.mark.parametrize("sees", ["tree", "chain"])
def test_more_sequences_than_are_staged(n_seq, sees):
    """Beyond 1024 every role reads the lengths and counts itself: ragged counts, absent and empty sequences, a long one."""
    rng = np.random.default_rng(53)
    lens = rng.integers(0, 40, (n_seq, 1))
    lens[rng.random((n_seq, 1)) < 0.1] = -1
    lens[400:520] = -1
    lens[n_seq - 3], lens[n_seq - 1] = 3000, -1
    count = rng.integers(0, 4, n_seq)
    count[n_seq - 3] = 3
    c = Tree(53, lens, 3, 2, 2, 16, sees=sees, count=count)
    out, lse = c.run()
    c.check(out, lse)
    again = c.run()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("n_seq,Hk", [(150, 1), (151, 1), (152, 1), (153, 1), (154, 1), (76, 2), (77, 2)])
def test_as_many_units_as_ctas(n_seq, Hk):
    """On both sides of the card's CTAs, units of one length and one that is longer."""
    for extra in (0, 300, 3000):
        lens = [[200 + 3 * (i % 5)] for i in range(n_seq)]
        lens[n_seq // 2][0] += extra
        c = Tree(36, lens, 1, 2 * Hk, Hk, 64, sees="chain")
        c.check(*c.run())


LONG_AMONG_SHORT = [[30 + i % 50] for i in range(50)] + [[20000]] + [[30 + i % 50] for i in range(50)]


@pytest.mark.parametrize("n_q,H", [(1, 2), (5, 8), (40, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_long_sequence_among_short_ones(n_q, H, dtype):
    """A unit in many parts beside whole ones, row tiles single and in pairs."""
    c = Tree(41, LONG_AMONG_SHORT, n_q, H, 1, 64, dtype=dtype)
    out, lse = c.run()
    c.check(out, lse)
    for _ in range(5):
        again = c.run()
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("fill", [0, 1, 255, 0x5a, None])
def test_a_workspace_of_any_content(fill):
    """Whatever the workspace holds before a call, and between calls."""
    c = Tree(42, LONG_AMONG_SHORT[40:], 3, 4, 1, 16)
    g = torch.Generator(device="cuda").manual_seed(5)
    first = None
    for i in range(4):
        if fill is None:
            c.ws.random_(0, 256, generator=g)
        else:
            c.ws.fill_(fill)
        out, lse = c.run()
        twice = c.run()  # (the workspace as the call left it)
        first = first if first is not None else out
        assert torch.equal(out, first) and torch.equal(twice[0], first)
    c.check(out, lse)


@pytest.mark.parametrize("n_q", [3, 40])
def test_a_workspace_on_any_16_byte_bound(n_q):
    """Cut units in a workspace that begins 0, 16 and 48 bytes past a bound of 256: the same bits, nothing written around it."""
    c = Tree(51, LONG_AMONG_SHORT[40:], n_q, 8, 1, 64)
    first, z = c.run()
    c.check(first, z)
    n = c.ws.numel()
    for at in (0, 16, 48):
        arena = torch.full((n + 512,), 0x5a, dtype=torch.uint8, device="cuda")
        at += 256 - arena.data_ptr() % 256
        c.ws = arena[at:at + n]
        out, lse = c.run()
        assert rps.rps_poll_device_status()[0] == rps.RPS_OK
        assert torch.equal(out, first) and torch.equal(lse, z)
        assert bool((arena[:at] == 0x5a).all()) and bool((arena[at + n:] == 0x5a).all())


@pytest.mark.parametrize("sees", ["tree", "chain"])
def test_the_largest_trees(sees):
    """1024 drafted tokens, 32 words a mask: eight pairs of row tiles; 64 with groups of 128 heads: 32 pairs of one token."""
    c = Tree(45, [[1100], [1024], [300]], 1024, 2, 1, 64, sees=sees, count=[1024, 1001, 300])
    c.check(*c.run())
    c = Tree(46, [[150], [64]], 64, 128, 1, 16, sees=sees)
    c.check(*c.run())


def test_two_calls_at_once():
    """On two streams, each with its workspace: as one after the other."""
    a, b = Tree(47, LONG_AMONG_SHORT, 3, 4, 1, 64), Tree(48, [[9000]] + [[70]] * 70, 40, 8, 1, 64)
    want = [x.run()[0].clone() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(w) for _ in range(6)] for w in want]
    torch.cuda.synchronize()
    for k in range(6):
        for x, s, out in zip((a, b), streams, outs):
            with torch.cuda.stream(s):
                x.run(out[k], lse=False, stream=s)
    torch.cuda.synchronize()
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert all(torch.equal(o, w) for w, out in zip(want, outs) for o in out)


def test_calls_of_other_shapes_and_graphs_share_a_workspace():
    a, b = Tree(43, LONG_AMONG_SHORT[40:], 3, 4, 1, 16), Tree(44, [[9000]] + [[70]] * 70, 2, 8, 1, 64, sees="chain")
    b.ws = a.ws = a.ws if a.ws.numel() >= b.ws.numel() else b.ws
    want = [x.run()[0].clone() for x in (a, b)]
    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.zeros_like(w) for w in want]
    for x, out in zip((a, b), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            x.run(out, lse=False)
        graphs.append(g)
    for i in (0, 1, 1, 0, 0, 1):
        outs[i].zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want[i])
        assert torch.equal((a, b)[1 - i].run()[0], want[1 - i])


def test_no_sequence_at_all():
    c = Tree(37, [[-1], [-1]], 3, 2, 1, 16)
    c.check(*c.run())
    c = Tree(37, [[40], [20]], 3, 2, 1, 16, count=[0, -1])
    c.check(*c.run())


def test_repeats_bit_for_bit_on_a_side_stream_and_from_a_graph():
    c = Tree(38, [[700], [129], [-1], [3000]], 40, 8, 2, 16)
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
    c.lens = np.array([[650], [-1], [-1], [500]])
    c.kv.length.copy_(torch.from_numpy(c.lens))
    out.fill_(7.0)
    g.replay()
    c.check(out, None)


@pytest.mark.parametrize("lens", [[[300], [290]], LONG_AMONG_SHORT])
def test_wait_timeout_is_reported_and_the_next_launch_works(lens):
    c = Tree(39, lens, 4, 2, 1, 16)
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
    c = Tree(40, [[40, 33]], 2, 4, 2, 16)
    args = lambda **kw: {**dict(q=c.dq, kv=c.kv, layer=0, out=torch.empty_like(c.dq), ws=c.ws, mask=c.mask, scale=0.1), **kw}
    for kw, err in ((dict(q=c.dq.float()), TypeError), (dict(out=torch.empty_like(c.dq, dtype=torch.float16)), TypeError),
                    (dict(q=c.dq[:, :1]), ValueError), (dict(out=c.dq[..., :64]), ValueError), (dict(out=c.dq[:, :, :1]), ValueError),
                    (dict(q=c.q), ValueError), (dict(mask=c.mask.long()), ValueError), (dict(mask=c.mask[:1]), ValueError),
                    (dict(n_tok=i32([1])), ValueError), (dict(lse=torch.empty(3, device="cuda")), ValueError),
                    (dict(ws=c.ws[:-1]), rps.RPSError), (dict(layer=1), rps.RPSError), (dict(scale=0.0), rps.RPSError),
                    (dict(q=c.dq.transpose(3, 4).contiguous().transpose(3, 4)), ValueError)):
        with pytest.raises(err):
            rps.rps_tree_attention_fwd(**args(**kw))
