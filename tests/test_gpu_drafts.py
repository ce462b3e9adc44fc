"""Drafted tokens: masks and positions from parents (rps_tree_masks), and the accepted path's
move to the front (rps_kv_keep_path), against the oracle (oracle/drafts.py). Integers and
moved rows: equal."""
import numpy as np
import pytest
import torch

from oracle import drafts
from oracle import kvcache as ok
from paper_2608_11742_gb300 import rps

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def parents(rng, n, kind):
    i = np.arange(n)
    return {"chain": i - 1, "roots": np.full(n, -1), "star": np.minimum(i - 1, 0),
            "random": np.array([rng.integers(-1, x) if x else -1 for x in i]),
            "wide": np.minimum(i - 1, i // 3 - 1 + rng.integers(0, 2, n))}[kind]


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 253, 1024])
@pytest.mark.parametrize("kind", ["chain", "roots", "star", "random", "wide"])
def test_masks(n, kind):
    rng = np.random.default_rng(n)
    n_seq = 5
    parent = np.stack([parents(rng, n, kind) for _ in range(n_seq)])
    count = np.array([n, max(1, n // 2), 0, n + 7, 1])
    length = rng.integers(2000, 9000, n_seq)
    for given, lens in ((None, None), (count, None), (count, length)):
        mask = torch.full((n_seq, n, -(-n // 32)), 7, dtype=torch.int32, device="cuda")
        pos = torch.full((n_seq, n), 7, dtype=torch.int32, device="cuda")
        rps.rps_tree_masks(i32(parent), mask, pos, None if given is None else i32(given), None if lens is None else i32(lens))
        assert rps.rps_poll_device_status()[0] == rps.RPS_OK
        for s in range(n_seq):
            m = n if given is None else min(n, count[s])
            sees, depth, _ = drafts.masks(parent[s], m)
            assert np.array_equal(mask[s, :m].cpu().numpy(), drafts.words(sees)[:m])
            assert np.array_equal(pos[s, :m].cpu().numpy(), depth[:m] + (0 if lens is None else lens[s] - m))
            assert bool((mask[s, m:] == 7).all()) and bool((pos[s, m:] == 7).all())
    alone = torch.zeros_like(mask)
    rps.rps_tree_masks(i32(parent), alone)
    assert np.array_equal(alone[0].cpu().numpy(), drafts.words(drafts.masks(parent[0], n)[0]))


def test_parents_out_of_range_are_flagged():
    parent = np.array([[-1, 0, 2, 5, -2, 3]])
    mask, pos = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((1, 6, 1), (1, 6)))
    rps.rps_tree_masks(i32(parent), mask, pos)
    assert rps.rps_poll_device_status() == (rps.RPS_ERR_DEVICE, rps.DEVERR_ROW_INDEX)
    assert mask.view(-1).tolist() == [1, 3, 4, 8, 16, 40] and pos.view(-1).tolist() == [0, 1, 0, 0, 0, 1]
    # behind the sequence's tokens anything may stand
    rps.rps_tree_masks(i32(parent), mask, pos, i32([2]))
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK


class Kept:
    def __init__(self, seed, lens, Hk, ps, layers, dtype=torch.bfloat16, tokens_first=False):
        rng = self.rng = np.random.default_rng(seed)
        lens = np.array(lens)
        pages = [0 if n <= 0 else -(-int(n) // ps) for n in lens]
        n_pages, at = sum(pages) + 3, 0
        table, place = np.full((len(lens), max(1, max(pages))), -1), rng.permutation(n_pages)
        for s, m in enumerate(pages):
            table[s, :m] = place[at:at + m]
            at += m
        ref = np.bincount(table[table >= 0].ravel(), minlength=n_pages)
        shape = (layers, n_pages, Hk, ps, 128)
        k, v = (torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype).cuda() for _ in range(2))
        if tokens_first:
            k, v = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (k, v))
        self.kv = rps.KvCacheBuf(k, v, i32(ref), i32(table[:, None]), i32(lens[:, None]))
        self.o = ok.Cache(ref, table, lens, ps, k.double().cpu().numpy(), v.double().cpu().numpy())

    def check(self, path, keep, n_q, count=None, status=0):
        new_len = torch.full((self.kv.n_seq,), 7, dtype=torch.int32, device="cuda")
        rps.rps_kv_keep_path(self.kv, i32(path), i32(keep), new_len, n_q, None if count is None else i32(count))
        assert rps.rps_poll_device_status()[1] == status
        want = drafts.keep_path(self.o, path, keep, n_q, count)
        assert self.o.err == status
        assert np.array_equal(new_len.cpu().numpy(), want)
        for got, x in ((self.kv.k, self.o.k), (self.kv.v, self.o.v)):
            assert np.array_equal(got.double().cpu().numpy(), x)
        assert np.array_equal(self.kv.length.cpu().numpy().ravel(), self.o.length)
        self.o.err = 0
        return new_len


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ps", [16, 64])
@pytest.mark.parametrize("Hk,layers", [(1, 1), (3, 2), (8, 5)])
def test_kept_paths(Hk, layers, ps, dtype):
    k = Kept(ps + Hk, [70, 33, -1, 200, 40, 64], Hk, ps, layers, dtype, Hk == 3)
    # everything, nothing, from the last one, every other, first ones
    path = np.zeros((6, 20), np.int64)
    path[0], path[1, 0], path[3, :10], path[4, :3], path[5, :7] = np.arange(20), 31, np.arange(3, 23, 2), [0, 1, 5], [1, 2, 3, 4, 28, 29, 30]
    k.check(path, np.array([20, 1, 5, 10, 3, 7]), 32)
    k.check(path, np.array([0, 1, 0, 2, 3, 0]), 32)


def test_long_paths_of_ragged_trees():
    k = Kept(3, [2100, 1500, 30], 2, 16, 1)
    path = np.stack([np.sort(k.rng.choice(n, 500, replace=False)) if n >= 500 else np.arange(500) for n in (1024, 700, 20)])
    k.check(path, np.array([500, 499, 20]), 1024, count=np.array([1024, 700, 20]))
    k.check(path, np.array([500, 1, 0]), 1024, count=np.array([1024, 700, -3]))


def test_paths_that_move_nothing():
    """Paths that do not ascend, leave the tree, or are longer than it, and sequences shorter than their tree."""
    k = Kept(4, [70, 70, 70, 70, 70, 20, 70, 70], 2, 16, 2)
    path = np.tile(np.array([2, 5, 9, 11]), (8, 1))
    path[0, 2], path[1, 1], path[2, 0], path[3, 3] = 5, 2, -1, 24
    k.check(path, np.array([4, 4, 4, 4, 5, 4, -1, 4]), 24, status=rps.DEVERR_ROW_INDEX)
    # entries past the kept ones are not looked at
    Kept(5, [70], 2, 16, 2).check(np.array([[2, 5, 9, 99]]), np.array([3]), 24)


def test_pages_that_are_shared_or_gone():
    k = Kept(6, [70, 70, 70], 2, 16, 2)
    shared = int(k.o.table[0, 3])
    k.kv.page_ref[shared] += 1
    k.o.ref[shared] += 1
    k.kv.table[1, 0, 4] = -1
    k.o.table[1, 4] = -1
    k.check(np.tile(np.array([3, 10, 18, 22]), (3, 1)), np.array([4, 4, 4]), 24, status=rps.DEVERR_SHARED | rps.DEVERR_PAGE)


def test_a_path_kept_from_a_graph():
    a, b = (Kept(7, [70, 33], 2, 16, 2) for _ in range(2))
    path, keep, new_len = i32([[2, 5], [0, 7]]), i32([2, 2]), torch.zeros(2, dtype=torch.int32, device="cuda")
    rps.rps_kv_keep_path(a.kv, path, keep, new_len, 8)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        rps.rps_kv_keep_path(b.kv, path, keep, new_len, 8)
    new_len.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.kv.k, b.kv.k) and torch.equal(a.kv.v, b.kv.v) and new_len.tolist() == [64, 27]


def test_refusals_of_the_binding():
    k = Kept(8, [70, 33], 2, 16, 2)
    path, keep = i32([[2, 5], [0, 7]]), i32([2, 2])
    for kw, err in ((dict(path=path[:1]), ValueError), (dict(path=path.long()), ValueError), (dict(n_keep=keep[:1]), ValueError),
                    (dict(new_len=torch.zeros(3, dtype=torch.int32, device="cuda")), ValueError), (dict(n_q=0), rps.RPSError),
                    (dict(n_q=1025), rps.RPSError), (dict(path=path.cpu()), ValueError), (dict(n_tok=i32([1])), ValueError)):
        with pytest.raises(err):
            rps.rps_kv_keep_path(**{**dict(kv=k.kv, path=path, n_keep=keep, new_len=None, n_q=8), **kw})
    parent, mask = i32(np.full((2, 40), -1)), torch.zeros((2, 40, 2), dtype=torch.int32, device="cuda")
    for kw, err in ((dict(parent=parent.long()), ValueError), (dict(mask=mask[:, :, :1]), ValueError), (dict(pos=mask), ValueError),
                    (dict(n_tok=i32([1])), ValueError), (dict(length=i32([1])), ValueError), (dict(mask=mask.cpu()), ValueError),
                    (dict(parent=i32(np.zeros((1, 2000)))), ValueError)):
        with pytest.raises(err):
            rps.rps_tree_masks(**{**dict(parent=parent, mask=mask), **kw})
