"""The K/V cache around a decoding step (rps.BranchCache with rps.Step): branches forked by the
pivots' list, their blocks written and attended, the step's winner committed, step after step,
also replayed from a graph; and caches whose offsets pass 32 bits."""
import numpy as np
import pytest
import torch

from oracle import kvcache as ok
from paper_2608_11742_gb300 import configs, rps, synth
from test_gpu_prefix_attention import D, EPS

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def normal(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)


class Run:
    """Two requests of 9 branches, a block of 16 tokens behind contexts of 21 and 48, two layers, 4 / 2 heads."""
    N_REQ, B, V, CTX, LAYERS, H, HK, PS = 2, 16, 4096, (21, 48), 2, 4, 2, 16

    def __init__(self, seed):
        self.rng = np.random.default_rng(seed)
        self.prm = configs.Params(10, 0.1, 0.0, 0.05, 0.1, 4, 2)
        nb = self.nb = 9
        self.step = rps.Step(self.N_REQ, self.B, self.V, self.prm, "cuda", torch.float32)
        self.cache = rps.BranchCache(self.LAYERS, 90, self.HK, self.PS, self.N_REQ, nb, 6, self.B, self.H, "cuda")
        self.ctx = i32(self.CTX)
        self.whole = self.ctx + self.B
        n = self.N_REQ * nb
        self.cache.kv.k.fill_(float("nan"))
        self.cache.kv.v.fill_(float("nan"))
        shape = tuple(self.cache.kv.k.shape)
        self.o = ok.Cache(np.zeros(shape[1]), np.full((n, 6), -1), np.full(n, -1), self.PS, np.full(shape, np.nan),
                          np.full(shape, np.nan))
        base = torch.full((self.N_REQ, nb), -1, dtype=torch.int32, device="cuda")
        base[:, 0] = self.ctx
        self.cache.resize(base)
        self.o.resize(base.cpu().numpy().ravel())
        for layer in range(self.LAYERS):
            self.write(layer, max(self.CTX))
        base[:, 0] = self.whole
        self.cache.resize(base)
        self.o.resize(base.cpu().numpy().ravel())

    def write(self, layer, n_new):
        k, v = (normal(self.rng, self.N_REQ, self.nb, n_new, self.HK, D) for _ in range(2))
        self.cache.write(layer, k.cuda(), v.cuda())
        self.o.write(layer, *[x.double().numpy().reshape(-1, n_new, self.HK, D) for x in (k, v)])

    def grown(self):
        return torch.where(self.cache.kv.length < 0, -1, self.whole[:, None]).int()

    def same_book(self):
        kv = self.cache.kv
        for got, want in ((kv.page_ref, self.o.ref), (kv.table, self.o.table), (kv.length, self.o.length)):
            assert np.array_equal(got.cpu().numpy().reshape(want.shape), want)

    def check_attention(self, layer):
        q = normal(self.rng, self.N_REQ, self.nb, self.B, self.H, D) * 2
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        scale = float(np.float32(D ** -0.5))
        self.cache.attend(layer, q.cuda(), out, self.ctx, scale)
        ref, mag, _ = ok.prefix_attention(q.double().numpy().reshape(-1, self.B, self.H, D), self.o, layer, scale, False)
        g = out.double().cpu().numpy().reshape(ref.shape)
        absent = np.isnan(ref)
        assert (g[absent] == 7.0).all()
        tol = EPS[torch.bfloat16] * (mag + np.abs(ref)) + 2.0 ** -12 * mag + 1e-6
        assert (np.abs(g - ref) <= tol)[~absent].all()


def test_steps_with_their_cache():
    """Four steps: the step's own pivots and winner drive the cache; its bookkeeping, its data (through the
    attention of every layer) and the counts at the end are the oracle's."""
    r = Run(41)
    mask_pos, mask_cnt = i32(np.tile(np.arange(r.B), (r.N_REQ, 1))), i32([r.B, r.B])
    logits = torch.empty((r.N_REQ, r.nb, r.B, r.V), dtype=torch.float32, device="cuda")
    winners = set()
    for step in range(4):
        synth.device_fill(logits, 100 + step, (0.4, 0.3, 0.3))
        r.step.run(logits, mask_pos, mask_cnt)
        valid = r.step.piv.branch_valid
        r.cache.fork(valid, r.ctx)
        r.o.fork_branches(r.nb, valid.cpu().numpy(), np.array(r.CTX))
        grown = r.grown()
        r.cache.resize(grown)
        r.o.resize(grown.cpu().numpy().ravel())
        r.same_book()
        for layer in range(r.LAYERS):
            r.write(layer, r.B)
            r.check_attention(layer)
        r.cache.commit(r.step.commit.winner)
        winner = r.step.commit.winner.cpu().numpy()
        winners |= set(winner.tolist())
        r.o.commit(r.nb, winner)
        if step == 2:
            r.cache.compact()
            assert r.o.compact() == int(r.cache.n_live)
        r.same_book()
        for layer in range(r.LAYERS):
            r.check_attention(layer)  # the bases alone
        assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert any(w >= 0 for w in winners), "no step committed a branch"


def test_a_step_of_the_cache_replayed():
    """fork, growth, write, attention and commit captured once and replayed: as the same calls made directly."""
    a, b = Run(42), Run(42)
    rng = np.random.default_rng(43)
    k, v, q = (normal(rng, 2, 9, 16, h, D).cuda() for h in (2, 2, 4))
    valid = torch.ones((2, 8), dtype=torch.uint8, device="cuda")
    valid[1, 3:] = 0
    winner, grown = i32([5, -1]), torch.full((2, 9), -1, dtype=torch.int32, device="cuda")
    grown[0], grown[1, :4] = int(a.whole[0]), int(a.whole[1])
    outs = [torch.zeros_like(q) for _ in range(2)]

    def step(r, out):
        r.cache.fork(valid, r.ctx)
        r.cache.resize(grown)
        r.cache.write(0, k, v)
        r.cache.attend(0, q, out, r.ctx, 0.1)
        r.cache.commit(winner)
        r.cache.compact()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(b, outs[1])
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(b, outs[1])
    step(a, outs[0])
    for _ in range(3):
        step(a, outs[0])
        g.replay()
    torch.cuda.synchronize()
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert torch.equal(outs[0], outs[1])
    for name in ("page_ref", "table", "length"):
        assert torch.equal(getattr(a.cache.kv, name), getattr(b.cache.kv, name))
    used = int(a.cache.n_live)
    same = lambda x, y: torch.equal(x[:, :used].contiguous().view(torch.int16), y[:, :used].contiguous().view(torch.int16))
    assert same(a.cache.kv.k, b.cache.kv.k) and same(a.cache.kv.v, b.cache.kv.v)


def test_offsets_beyond_32_bits():
    """A cache whose pages lie beyond 2^32 bytes and 2^31 elements: written, copied and attended as in a small one."""
    layers, heads, ps, pages = 2, 8, 64, 20000  # 2.6 G elements, 5.2 GB each of keys and values
    big = rps.KvCacheBuf.alloc(layers, pages, heads, ps, 1, 2, 3, "cuda")
    small = rps.KvCacheBuf.alloc(layers, 8, heads, ps, 1, 2, 3, "cuda")
    rng = np.random.default_rng(44)
    at = {0: [19990, 17, 19999], 1: [19990, 19998, 16500]}
    k, v = (normal(rng, 1, 2, 150, heads, D).cuda() for _ in range(2))
    # the 64 shared tokens are put into their page directly: no sequence may write a page that two hold
    first_k, first_v = (x[0, 0, :64].transpose(0, 1) for x in (k, v))
    q = normal(rng, 1, 2, 5, 16, D).cuda()
    outs = []
    for kv, ids in ((big, at), (small, {0: [6, 1, 7], 1: [6, 2, 3]})):
        kv.table.copy_(i32([[ids[0], ids[1]]]))
        kv.length.copy_(i32([[150, 150]]))
        for row in ids.values():
            kv.page_ref[torch.tensor(row)] += 1
        kv.k[1, ids[0][0]], kv.v[1, ids[0][0]] = first_k, first_v
        rps.rps_kv_write(kv, 1, k[:, :, 64:], v[:, :, 64:])
        out = torch.zeros_like(q)
        ws = torch.empty(rps.rps_prefix_attention_workspace_bytes(kv, 5, 16), dtype=torch.uint8, device="cuda")
        rps.rps_prefix_attention_fwd(q, kv, 1, out, ws, i32([64]), 0.1)
        outs.append(out)
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert torch.equal(outs[0], outs[1]) and bool(outs[0].abs().sum() > 0)
    rps.rps_kv_copy_pages(big, big, i32([19999, 17]), i32([19997, 19996]))
    # (22 tokens of the third page are written; what lies behind them is copied as it is)
    assert torch.equal(big.k[1, 19997, :, :22], small.k[1, 7, :, :22])
    assert torch.equal(big.k[:, 19997].view(torch.int16), big.k[:, 19999].view(torch.int16))
    assert torch.equal(big.v[1, 19996], small.v[1, 1])
