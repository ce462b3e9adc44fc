"""Pages of the K/V cache (rps_kv_*) against the oracle (oracle/kvcache.py): runs of
forks, growth, commits, frees, writes, compactions and copies, bookkeeping and every
bit of the data compared after each call. Data are random bit patterns (NaN among
them): the calls move them and compute nothing."""
import numpy as np
import pytest
import torch

from oracle import kvcache as ok
from paper_2608_11742_gb300 import rps

pytestmark = pytest.mark.gpu

D = 128


def bits(rng, shape):
    return rng.integers(-2 ** 15, 2 ** 15, shape, dtype=np.int64).astype(np.int16)


def dev16(a, dtype=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().view(dtype)


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def poll():
    status, detail = rps.rps_poll_device_status()
    assert status in (rps.RPS_OK, rps.RPS_ERR_DEVICE)
    return detail


class Pair:
    """A cache on the device and its oracle."""

    def __init__(self, seed, layers, pages, heads, ps, n_req, nb, width, dtype=torch.bfloat16, tokens_first=False):
        self.rng = np.random.default_rng(seed)
        self.n_req, self.nb, self.width, self.ps = n_req, nb, width, ps
        self.kv = rps.KvCacheBuf.alloc(layers, pages, heads, ps, n_req, nb, width, "cuda", dtype)
        if tokens_first:  # [pages][tokens][heads] in memory
            for name in ("k", "v"):
                t = torch.empty((layers, pages, ps, heads, D), dtype=dtype, device="cuda").transpose(2, 3)
                setattr(self.kv, name, t)
        k, v = bits(self.rng, (layers, pages, heads, ps, D)), bits(self.rng, (layers, pages, heads, ps, D))
        self.kv.k.view(torch.int16).copy_(torch.from_numpy(k))
        self.kv.v.view(torch.int16).copy_(torch.from_numpy(v))
        n = n_req * nb
        self.o = ok.Cache(np.zeros(pages), np.full((n, width), -1), np.full(n, -1), ps, k, v)
        # (exactly the bytes asked for, inside a larger buffer that must stay as it is)
        size = rps.rps_kv_workspace_bytes(self.kv)
        self.guard = torch.full((size + 512,), 77, dtype=torch.uint8, device="cuda")
        self.ws = self.guard[256:256 + size]

    def check(self, what):
        detail = poll()
        assert detail == self.o.err, f"{what}: error bits {detail:#x}, expected {self.o.err:#x}"
        self.o.err = 0
        for name, got, want in (("len", self.kv.length, self.o.length), ("table", self.kv.table, self.o.table),
                                ("ref", self.kv.page_ref, self.o.ref)):
            g = got.cpu().numpy().reshape(want.shape)
            assert np.array_equal(g, want), f"{what}: {name} differs at {np.argwhere(g != want)[:4].tolist()}"
        for name, got, want in (("k", self.kv.k, self.o.k), ("v", self.kv.v, self.o.v)):
            g = got.contiguous().view(torch.int16).cpu().numpy()
            assert np.array_equal(g, want), f"{what}: {name} differs at {np.argwhere(g != want)[:4].tolist()}"
        g = self.guard.cpu().numpy()
        assert (g[:256] == 77).all() and (g[-256:] == 77).all(), f"{what}: wrote outside the workspace"

    def resize(self, new_len):
        rps.rps_kv_resize(self.kv, i32(new_len), self.ws)
        self.o.resize(list(new_len))
        self.check(f"resize {list(new_len)[:8]}")

    def reorder(self, src, keep=None):
        rps.rps_kv_reorder(self.kv, i32(src), self.ws, None if keep is None else i32(keep))
        self.o.reorder(list(src), keep)
        self.check(f"reorder {list(src)[:8]}")

    def fork(self, valid, ctx):
        rps.rps_kv_fork_branches(self.kv, torch.from_numpy(valid.astype(np.uint8)).cuda(),
                                 None if ctx is None else i32(ctx), self.ws)
        self.o.fork_branches(self.nb, valid, ctx)
        self.check("fork")

    def commit(self, winner):
        rps.rps_kv_commit(self.kv, i32(winner), self.ws)
        self.o.commit(self.nb, list(winner))
        self.check(f"commit {list(winner)[:8]}")

    def write(self, layer, n_new, heads_first=False):
        n, h = self.n_req * self.nb, self.o.k.shape[2]
        new = [bits(self.rng, (n, n_new, h, D)) for _ in range(2)]
        shape = (self.n_req, self.nb, n_new, h, D)
        ts = [dev16(x, self.kv.k.dtype).view(shape) for x in new]
        if heads_first:
            ts = [t.transpose(2, 3).contiguous().transpose(2, 3) for t in ts]
        rps.rps_kv_write(self.kv, layer, ts[0], ts[1])
        self.o.write(layer, *new)
        self.check(f"write {n_new}")

    def compact(self):
        n_live = torch.zeros(1, dtype=torch.int32, device="cuda")
        rps.rps_kv_compact(self.kv, n_live, self.ws)
        want = self.o.compact()
        self.check("compact")
        assert int(n_live) == want


@pytest.mark.parametrize("layers,pages,heads,ps,n_req,nb,width,dtype,tokens_first", [
    (1, 40, 1, 16, 1, 3, 6, torch.bfloat16, False),
    (2, 64, 3, 16, 2, 5, 9, torch.float16, True),
    (1, 70, 2, 32, 3, 4, 5, torch.bfloat16, True),
    (3, 50, 2, 64, 4, 3, 4, torch.float16, False),
    (1, 30, 1, 256, 5, 2, 3, torch.bfloat16, True),
    (1, 700, 1, 16, 37, 9, 7, torch.bfloat16, False),   # 333 sequences: more than a block has warps
    (1, 3000, 1, 16, 60, 9, 12, torch.float16, False),  # a cluster's share for each of its blocks
])
def test_random_runs(layers, pages, heads, ps, n_req, nb, width, dtype, tokens_first):
    p = Pair(7, layers, pages, heads, ps, n_req, nb, width, dtype, tokens_first)
    rng, n, most = np.random.default_rng(8), n_req * nb, width * ps
    for step in range(30):
        op = rng.integers(0, 7)
        if op <= 1:  # some grow, some shrink, some end, some stay; sometimes beyond the pages there are
            new = np.where(rng.random(n) < 0.5, rng.integers(-1, most + 1, n), p.o.length)
            new = np.where(rng.random(n) < 0.3, np.minimum(most, p.o.length + rng.integers(0, 4, n)), new)
            if rng.random() < 0.7:
                new = np.minimum(new, max(1, pages * ps // n))
            p.resize(new)
        elif op == 2:
            src = rng.integers(-1, n, n)
            p.reorder(src, rng.integers(-1, most + 1, n) if rng.random() < 0.5 else None)
        elif op == 3:
            p.fork(rng.random((n_req, nb - 1)) < 0.7, rng.integers(0, most, n_req) if rng.random() < 0.8 else None)
        elif op == 4:
            p.commit(rng.integers(-3, nb - 1, n_req))
        elif op == 5:
            p.write(int(rng.integers(0, layers)), int(rng.integers(1, 2 * ps // 3)), bool(rng.integers(0, 2)))
        else:
            p.compact()


def test_more_sequences_than_fit_a_blocks_shared_memory():
    p = Pair(17, 1, 6000, 1, 16, 3000, 3, 2)
    rng = np.random.default_rng(18)
    p.resize(rng.integers(-1, 12, 9000))
    p.resize(np.where(p.o.length < 6, -1, p.o.length + 9))
    p.commit(rng.integers(-1, 2, 3000))
    p.compact()


def test_lookahead_cycle():
    """Context written, branches forked from it, grown by their block (the shared last page copied for each),
    written, the winner committed: the base then holds the winner's block after its own context."""
    p = Pair(9, 2, 80, 2, 16, 3, 5, 8)
    ctx, block = np.array([37, 48, 5]), 20
    base = lambda v: np.where(np.arange(15) % 5 == 0, np.repeat(v, 5), -1)
    p.resize(base(ctx))
    p.write(0, 48)
    p.write(1, 48)
    p.resize(base(ctx + block))
    p.write(0, block)
    valid = np.array([[1, 1, 0, 1], [0, 0, 0, 0], [1, 1, 1, 1]]) > 0
    p.fork(valid, ctx)
    assert p.o.length.reshape(3, 5)[0].tolist() == [57, 37, 37, -1, 37]
    p.resize(np.where(p.o.length < 0, -1, np.repeat(ctx + block, 5)))
    p.write(0, block)
    p.write(1, block)
    p.commit([3, -1, 0])
    p.compact()
    held = int((p.o.ref > 0).sum())
    assert (p.o.ref[:held] == 1).all() and (p.o.ref[held:] == 0).all()


def test_grown_to_the_last_page_and_not_beyond():
    p = Pair(10, 1, 6, 1, 16, 1, 4, 6)
    p.resize([32, 16, 0, -1])
    p.resize([48, 49, 1, 16])     # 1 + 3 wanted, 3 free: the second does not fit, nor do those after it
    p.resize([48, 16, 17, -1])    # the two that are left
    p.resize([-1, 16, 17, 96])    # 3 given back in the same call, 6 wanted
    p.resize([-1, 16, 17, 48])
    p.resize([97, 16, 17, 48])    # beyond the table's width
    p.resize([-1, -1, -1, -1])
    assert (p.o.ref == 0).all()


def test_every_holder_of_a_shared_last_page_copies_it():
    p = Pair(11, 2, 12, 2, 16, 1, 3, 4)
    p.resize([20, -1, -1])
    p.write(0, 20)
    p.reorder([0, 0, 0])
    assert p.o.ref.max() == 3
    p.write(1, 2)                  # the page is shared: left out, reported
    p.resize([21, 25, 33])
    assert p.o.ref[p.o.table[0, 1]] == 1
    p.write(1, 2)


def test_bad_bookkeeping_is_reported_and_stays_inside():
    """Ids outside the cache, lengths beyond the table and sources outside the sequences: the error word says
    so, nothing outside is touched."""
    p = Pair(12, 1, 10, 1, 16, 1, 4, 3)
    p.resize([40, 20, -1, 5])
    p.reorder([4, -2, 0, 3])       # two sources that do not exist
    p.commit([7])
    p.resize([40, 20, -1, 5])
    p.kv.table[0, 0, 1] = 10
    p.kv.table[0, 1, 0] = -5
    p.o.table[0, 1], p.o.table[1, 0] = 10, -5
    p.write(0, 40)
    p.reorder([0, 1, 0, 1])
    p.resize([-1, -1, -1, -1])
    p.kv.length[0, 2] = 49
    rps.rps_kv_write(p.kv, 0, *[torch.zeros((1, 4, 1, 1, D), dtype=torch.bfloat16, device="cuda")] * 2)
    assert poll() & rps.DEVERR_PAGE


@pytest.mark.parametrize("heads,ps,n,tokens", [(1, 16, 1, (False, True)), (3, 64, 7, (True, True)),
                                               (2, 256, 5, (True, False)), (5, 16, 23, (False, False))])
def test_copy_pages(heads, ps, n, tokens):
    a, b = (Pair(13 + i, 2, 30 + 3 * i, heads, ps, 1, 1, 2, tokens_first=t) for i, t in enumerate(tokens))
    rng = np.random.default_rng(15)
    src, dst = rng.integers(0, 30, n), rng.permutation(33)[:n]
    rps.rps_kv_copy_pages(a.kv, b.kv, i32(src), i32(dst))
    for x, y in ((a.o.k, b.o.k), (a.o.v, b.o.v)):
        y[:, dst] = x[:, src]
    b.check("copy")
    rps.rps_kv_copy_pages(a.kv, b.kv, i32([30, 3, -1, 5]), i32([1, 33, 2, 6]))  # three ids outside
    b.o.k[:, 6], b.o.v[:, 6] = a.o.k[:, 5], a.o.v[:, 5]
    b.o.err = rps.DEVERR_PAGE
    b.check("copy of ids outside")
    rps.rps_kv_copy_pages(a.kv, b.kv, i32([]), i32([]))
    b.check("copy of nothing")


def test_on_a_side_stream_and_replayed_from_a_graph():
    p = Pair(16, 1, 40, 2, 16, 2, 3, 5)
    side = torch.cuda.Stream()
    valid = torch.ones((2, 2), dtype=torch.uint8, device="cuda")
    ctx, grown, winner = i32([20, 9]), i32([[40, 40, 40], [29, 29, 29]]), i32([1, -1])
    start = i32([[20, -1, -1], [9, -1, -1]])
    new = [dev16(bits(p.rng, (2, 3, 20, 2, D))) for _ in range(2)]
    torch.cuda.synchronize()

    def cycle(stream=None):
        rps.rps_kv_resize(p.kv, start, p.ws, stream)
        rps.rps_kv_fork_branches(p.kv, valid, ctx, p.ws, stream)
        rps.rps_kv_resize(p.kv, grown, p.ws, stream)
        rps.rps_kv_write(p.kv, 0, new[0], new[1], stream)
        rps.rps_kv_commit(p.kv, winner, p.ws, stream)
        rps.rps_kv_compact(p.kv, None, p.ws, stream)

    def oracle():
        p.o.resize([20, -1, -1, 9, -1, -1])
        p.o.fork_branches(3, np.ones((2, 2)), [20, 9])
        p.o.resize([40, 40, 40, 29, 29, 29])
        p.o.write(0, *[x.view(torch.int16).cpu().numpy().reshape(6, 20, 2, D) for x in new])
        p.o.commit(3, [1, -1])
        p.o.compact()

    cycle(side)
    oracle()
    side.synchronize()
    p.check("on a side stream")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        cycle(side)
    for _ in range(3):
        g.replay()
        oracle()
    torch.cuda.synchronize()
    p.check("replayed")


@pytest.mark.parametrize("n_req,nb", [(2, 3), (70, 4)])  # one block, a cluster
def test_sequences_of_many_pages(n_req, nb):
    """Few and many pages taken and given back side by side (a thread alone, a warp together), partial last pages
    shared and copied on the way."""
    n, width = n_req * nb, 90
    p = Pair(31, 1, n * 60, 1, 16, n_req, nb, width)
    rng = np.random.default_rng(32)
    for k in range(6):
        p.resize(rng.choice([-1, 0, 5, 16 * 32, 16 * 33, 16 * 34 - 3, 600, 16 * width], n, p=[.1, .1, .2, .2, .1, .1, .1, .1]))
        if k % 2 == 0:
            p.fork(rng.random((n_req, nb - 1)) < 0.7, None)
            p.resize(np.where(p.o.length > 0, np.minimum(p.o.length + rng.choice([1, 40, 16 * 40], n), 16 * width), p.o.length))
    p.resize(np.full(n, -1))
    assert (p.o.ref == 0).all()


@pytest.mark.parametrize("heads,n_new,tokens_first", [(3, 171, False), (3, 400, True), (28, 19, True), (1, 1100, False),
                                                      (600, 2, True), (600, 3, False)])
def test_writes_of_more_rows_than_a_block_takes(heads, n_new, tokens_first):
    """512 rows a block: blocks that begin and end inside a token's heads, more heads than rows of a block."""
    ps, layers = 16, 1
    width = -(-(n_new + 9) // ps)
    p = Pair(33, layers, 2 * width, heads, ps, 1, 2, width, tokens_first=tokens_first)
    p.resize([n_new + 9, n_new - 2])
    p.write(0, n_new)
    p.write(0, n_new, heads_first=True)


def test_writes_with_one_branch_and_odd_strides():
    """One branch: sequences lie at the request's stride, whatever the branch's is; rows wider than they are read."""
    p = Pair(34, 1, 12, 2, 16, 3, 1, 4)
    p.resize([20, 7, 33])
    wide = [dev16(bits(p.rng, (3, 5, 2, D + 24))) for _ in range(2)]
    k, v = (w[:, None, :, :, :D] for w in wide)
    rps.rps_kv_write(p.kv, 0, k, v)
    p.o.write(0, *[x[:, 0].contiguous().view(torch.int16).cpu().numpy() for x in (k, v)])
    p.check("write")


def test_refusals_of_the_binding():
    p = Pair(35, 1, 12, 2, 16, 2, 2, 3)
    p.resize([16, -1, 16, -1])
    ok_new = torch.zeros((2, 2, 4, 2, D), dtype=torch.bfloat16, device="cuda")
    ws, kv = p.ws, p.kv
    four, two = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.full((2,), -1, dtype=torch.int32, device="cuda")
    valid = torch.zeros((2, 1), dtype=torch.uint8, device="cuda")
    refused = [
        lambda: rps.rps_kv_write(kv, 0, ok_new[:, :, :, :1], ok_new[:, :, :, :1]),              # heads
        lambda: rps.rps_kv_write(kv, 0, ok_new, ok_new[:, :, :3]),                              # shapes differ
        lambda: rps.rps_kv_write(kv, 0, ok_new.half(), ok_new.half()),                          # type
        lambda: rps.rps_kv_write(kv, 0, ok_new.cpu(), ok_new.cpu()),                            # device
        lambda: rps.rps_kv_write(kv, 0, ok_new, ok_new.transpose(2, 3).contiguous().transpose(2, 3)),  # strides differ
        lambda: rps.rps_kv_write(kv, 0, ok_new.transpose(0, 1), ok_new.transpose(0, 1)),        # requests inside branches
        lambda: rps.rps_kv_write(kv, 1, ok_new, ok_new),                                        # layer
        lambda: rps.rps_kv_write(kv, -1, ok_new, ok_new),
        lambda: rps.rps_kv_resize(kv, four.long(), ws),
        lambda: rps.rps_kv_resize(kv, four[:3], ws),
        lambda: rps.rps_kv_resize(kv, four.cpu(), ws),
        lambda: rps.rps_kv_resize(kv, four, ws[:-1]),
        lambda: rps.rps_kv_reorder(kv, four, ws, four[:2]),
        lambda: rps.rps_kv_fork_branches(kv, valid.int(), None, ws),
        lambda: rps.rps_kv_fork_branches(kv, valid, four, ws),
        lambda: rps.rps_kv_commit(kv, four, ws),
        lambda: rps.rps_kv_compact(kv, two, ws),
        lambda: rps.rps_kv_copy_pages(kv, kv, four, two),
        lambda: rps.rps_kv_copy_pages(kv, rps.KvCacheBuf.of_pages(kv.k.half(), kv.v.half()), two, two),
    ]
    for i, call in enumerate(refused):
        with pytest.raises((ValueError, TypeError, rps.RPSError)):
            call()
            pytest.fail(f"call {i} was not refused")
    p.check("refused calls")


def test_copies_of_the_buffer_object():
    """copy.copy shares the tensors, a deep copy and a pickle have their own; replaced tensors are used."""
    import copy
    import pickle
    p = Pair(36, 1, 8, 1, 16, 1, 2, 3)
    p.resize([20, 3])
    shared, own, loaded = copy.copy(p.kv), copy.deepcopy(p.kv), pickle.loads(pickle.dumps(p.kv))
    before = p.kv.length.clone()
    rps.rps_kv_resize(own, i32([5, -1]), p.ws)
    rps.rps_kv_resize(loaded, i32([40, 40]), p.ws)
    p.check("other buffers' calls")
    assert own.length.tolist() == [[5, -1]] and loaded.length.tolist() == [[40, 40]]
    assert torch.equal(p.kv.length, before)
    rps.rps_kv_resize(shared, i32([17, 3]), p.ws)
    p.o.resize([17, 3])
    p.check("a shallow copy's call")
    p.kv.length = p.kv.length.clone()  # the struct is built anew
    p.resize([1, 30])
    assert shared.length.tolist() == [[17, 3]]
