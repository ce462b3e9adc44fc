"""Drafted trees around the paged cache (rps.BranchCache with tree=True), as they are used together:
masks and positions from parents, pages for the tokens, keys appended with their norms and
positions, the attention under the masks, the accepted path kept; step after step, and replayed
from a graph. Tolerances: those of the single operators' tests."""
import numpy as np
import pytest
import torch

from oracle import drafts
from oracle import kvcache as ok
from paper_2608_11742_gb300 import rps
from test_gpu_prefix_attention import D, EPS
from test_gpu_rope import EPS as NORM_EPS, AMP, check, i32, make_rope, normal

pytestmark = pytest.mark.gpu


class Run:
    """Three sequences (two requests' worth of branches would be more sequences: none is shared here), trees of up to
    12 tokens, two layers, 6 / 2 heads, pages of 16."""
    N, N_Q, H, HK, PS, LAYERS, WIDTH = 3, 12, 6, 2, 16, 2, 8

    def __init__(self, seed, dtype=torch.bfloat16):
        self.rng = np.random.default_rng(seed)
        self.dtype = dtype
        self.cache = rps.BranchCache(self.LAYERS, 30, self.HK, self.PS, self.N, 1, self.WIDTH, self.N_Q, self.H, "cuda", dtype,
                                     tree=True)
        kv = self.cache.kv
        kv.k.fill_(float("nan"))
        kv.v.fill_(float("nan"))
        shape = tuple(kv.k.shape)
        self.o = ok.Cache(np.zeros(shape[1]), np.full((self.N, self.WIDTH), -1), np.full(self.N, -1), self.PS, np.full(shape, np.nan),
                          np.full(shape, np.nan))
        self.rope, self.freq, (self.wq, self.wk) = make_rope(self.rng, D, 64, dtype)
        self.mask = torch.zeros((self.N, 1, self.N_Q, 1), dtype=torch.int32, device="cuda")
        self.pos = torch.zeros((self.N, 1, self.N_Q), dtype=torch.int32, device="cuda")

    def tokens(self):
        rows = normal(self.rng, self.dtype, self.N, 1, self.N_Q, self.H + 2 * self.HK, D)
        return rows[..., :self.H, :], rows[..., self.H:self.H + self.HK, :], rows[..., self.H + self.HK:, :]

    def same_book(self):
        kv = self.cache.kv
        for got, want in ((kv.page_ref, self.o.ref), (kv.table, self.o.table), (kv.length, self.o.length)):
            assert np.array_equal(got.cpu().numpy().reshape(want.shape), want)

    def step(self, parent, count, path, keep):
        """One step on the cache and on the oracle; ctx: tokens before it."""
        c, n_q = self.cache, self.N_Q
        ctx = np.maximum(self.o.length, 0)
        grown = np.where(count > 0, ctx + count, self.o.length)
        c.resize(i32(grown[:, None]))
        self.o.resize(grown)
        rps.rps_tree_masks(i32(parent[:, None]), self.mask, self.pos, i32(count), c.kv.length)
        sees = np.stack([drafts.masks(parent[s], int(count[s]))[0] for s in range(self.N)])
        depth = np.stack([drafts.masks(parent[s], int(count[s]))[1] for s in range(self.N)])
        for layer in range(self.LAYERS):
            q, k, v = self.tokens()
            q_out, out = (torch.full(q.shape, 7.0, dtype=self.dtype, device="cuda") for _ in range(2))
            c.append(layer, self.rope, k, v, q, q_out, i32(count), self.pos)
            c.attend_tree(layer, q_out, out, self.mask, D ** -0.5, i32(count))
            assert rps.rps_poll_device_status()[0] == rps.RPS_OK
            for s, i, token, page in drafts.append_places(self.o, n_q, count):
                at = int(ctx[s] + depth[s, i])
                check(q_out[s, 0, i][None], q[s, 0, i][None], self.wq, self.freq, False, np.array([at]), self.dtype)
                check(c.kv.k[layer, page, :, token % self.PS][None], k[s, 0, i][None], self.wk, self.freq, False, np.array([at]), self.dtype)
                # (the attention is checked on the keys that the cache holds)
                self.o.k[layer, page, :, token % self.PS] = c.kv.k[layer, page, :, token % self.PS].double().cpu().numpy()
                self.o.v[layer, page, :, token % self.PS] = v[s, 0, i].double().cpu().numpy()
            ref, mag, _ = drafts.tree_attention(q_out[:, 0].double().cpu().numpy(), self.o, layer, float(np.float32(D ** -0.5)), count, sees)
            g = out[:, 0].double().cpu().numpy()
            absent = np.isnan(ref)
            assert (g[absent] == 7.0).all()
            tol = EPS[self.dtype] * (mag + np.abs(ref)) + 2.0 ** -12 * mag + 1e-6
            assert (np.abs(g - ref) <= tol)[~absent].all()
        c.keep_path(i32(path), i32(keep), n_q, i32(count))
        new_len = drafts.keep_path(self.o, path, keep, n_q, count)
        self.o.resize(new_len)
        self.same_book()
        for got, want in ((c.kv.k, self.o.k), (c.kv.v, self.o.v)):
            for s in range(self.N):
                for t in range(max(0, int(self.o.length[s]))):
                    p = self.o.table[s, t // self.PS]
                    assert np.array_equal(got[:, p, :, t % self.PS].double().cpu().numpy(), want[:, p, :, t % self.PS])


def random_step(rng, n, n_q, kind):
    parent = np.array([[rng.integers(-1, i) if i else -1 for i in range(n_q)] for _ in range(n)])
    count = np.array([n_q, n_q // 2, 1]) if kind else np.full(n, n_q)
    path, keep = np.zeros((n, n_q), np.int64), np.zeros(n, np.int64)
    for s in range(n):
        node = int(rng.integers(0, count[s]))  # the accepted leaf, and its ancestors
        chain = []
        while node >= 0:
            chain.append(node)
            node = parent[s, node]
        keep[s] = len(chain)
        path[s, :keep[s]] = chain[::-1]
    return parent, count, path, keep


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_steps_of_drafted_trees(dtype):
    """Prompts as chains, then five steps of trees of which a path is kept: lengths, pages, keys and every layer's
    attention are the oracle's."""
    r = Run(51, dtype)
    chain = np.tile(np.arange(-1, r.N_Q - 1), (r.N, 1))
    everything = np.tile(np.arange(r.N_Q), (r.N, 1))
    r.step(chain, np.array([12, 7, 3]), everything, np.array([12, 7, 3]))
    for i in range(5):
        r.step(*random_step(r.rng, r.N, r.N_Q, i % 2))
    assert min(r.o.length) > 3


def test_a_step_replayed():
    """Growth, masks, append, attention and the kept path captured once and replayed on new parents: as the calls made
    directly."""
    a, b = Run(52), Run(52)
    steps = [random_step(np.random.default_rng(60 + i), 3, 12, i % 2) for i in range(4)]
    rows = [tuple(x.clone() for x in a.tokens()) for _ in range(4)]
    outs = []
    grid = {k: torch.zeros(s, dtype=torch.int32, device="cuda") for k, s in (("parent", (3, 1, 12)), ("count", (3, 1)), ("path", (3, 12)),
                                                                            ("keep", (3,)), ("grown", (3, 1)))}
    q, k, v = (torch.zeros_like(x) for x in rows[0])
    q_out, out = torch.zeros_like(q), torch.zeros_like(q)

    def calls(r):
        torch.add(r.cache.kv.length.clamp(min=0), grid["count"], out=grid["grown"])
        r.cache.resize(grid["grown"])
        rps.rps_tree_masks(grid["parent"], r.mask, r.pos, grid["count"], r.cache.kv.length)
        for layer in range(r.LAYERS):
            r.cache.append(layer, r.rope, k, v, q, q_out, grid["count"], r.pos)
            r.cache.attend_tree(layer, q_out, out, r.mask, 0.1, grid["count"])
        r.cache.keep_path(grid["path"], grid["keep"], 12, grid["count"])

    def load(i):
        for name, x in zip(("parent", "count", "path", "keep"), steps[i]):
            grid[name].copy_(torch.from_numpy(x.astype(np.int32)).view(grid[name].shape))
        for to, x in zip((q, k, v), rows[i]):
            to.copy_(x)

    # every run: its first step directly, the others directly or from the graph
    for r, replayed in ((a, False), (b, True)):
        load(0)
        calls(r)
        torch.cuda.synchronize()
        if replayed:
            side = torch.cuda.Stream()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                calls(r)
        got = []
        for i in range(1, 4):
            load(i)
            out.fill_(7.0)
            g.replay() if replayed else calls(r)
            torch.cuda.synchronize()
            got.append(out.clone())
        outs.append(got)
        assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    assert torch.equal(a.cache.kv.length, b.cache.kv.length) and torch.equal(a.cache.kv.table, b.cache.kv.table)


def test_branches_that_share_their_context():
    """Trees on the branches of a request: the shared pages are read, the branches' own are written."""
    rng = np.random.default_rng(53)
    cache = rps.BranchCache(1, 20, 2, 16, 1, 3, 6, 5, 4, "cuda", tree=True)
    rope, freq, (wq, wk) = make_rope(rng, D, 128, torch.bfloat16)
    cache.resize(i32([[40, -1, -1]]))
    k, v = normal(rng, torch.bfloat16, 1, 3, 40, 2, D), normal(rng, torch.bfloat16, 1, 3, 40, 2, D)
    cache.append(0, rope, k, v)
    cache.fork(torch.ones((1, 2), dtype=torch.uint8, device="cuda"), i32([37]))
    cache.resize(i32([[45, 42, 42]]))
    q, k2, v2 = (normal(rng, torch.bfloat16, 1, 3, 5, h, D) for h in (4, 2, 2))
    out = torch.zeros_like(q)
    cache.append(0, rope, k2, v2, q, q)
    cache.attend_tree(0, q, out, None, 0.1)
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    # a branch alone, its keys in pages of its own
    for b, ctx in enumerate((40, 37, 37)):
        alone = rps.BranchCache(1, 5, 2, 16, 1, 1, 6, 5, 4, "cuda", tree=True)
        alone.resize(i32([[ctx]]))
        alone.append(0, rope, k[:, :1, :ctx], v[:, :1, :ctx])
        alone.resize(i32([[ctx + 5]]))
        alone.append(0, rope, k2[:, b:b + 1], v2[:, b:b + 1])
        one = torch.zeros_like(q[:, :1])
        alone.attend_tree(0, q[:, b:b + 1], one, None, 0.1)
        assert torch.equal(one[0, 0], out[0, b]), b


def test_a_cache_made_without_trees_refuses():
    cache = rps.BranchCache(1, 5, 2, 16, 1, 1, 6, 5, 4, "cuda")
    q = torch.zeros((1, 1, 5, 4, D), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        cache.attend_tree(0, q, q.clone(), None, 0.1)


def test_offsets_beyond_32_bits():
    """A tree over pages beyond 2^32 bytes: as in a small cache."""
    rng = np.random.default_rng(54)
    outs = []
    q, k, v = (normal(rng, torch.bfloat16, 1, 1, 40, h, D) for h in (16, 8, 8))
    for pages, ids in ((20000, [19990, 17, 19999]), (8, [6, 1, 7])):
        kv = rps.KvCacheBuf.alloc(2, pages, 8, 64, 1, 1, 3, "cuda")
        kv.table.copy_(i32([[ids]]))
        kv.length.fill_(140)
        for p in ids:
            kv.page_ref[p] = 1
            kv.k[1, p] = kv.v[1, p] = 0.25
        rps.rps_kv_append(kv, 1, None, k, v)
        out = torch.zeros_like(q)
        ws = torch.empty(rps.rps_tree_attention_workspace_bytes(kv, 40, 16), dtype=torch.uint8, device="cuda")
        rps.rps_tree_attention_fwd(q, kv, 1, out, ws, None, 0.1)
        rps.rps_kv_keep_path(kv, i32([[3, 39]]), i32([2]), None, 40)
        torch.cuda.synchronize()
        outs.append((out, kv.k[1, ids[1], :, 36:38].clone()))
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and bool(outs[0][0].abs().sum() > 0)
