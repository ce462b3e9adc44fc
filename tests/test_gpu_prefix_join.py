"""Attention over the paged K/V cache whose row tiles are cut: every row tile that has several
parts is joined, whatever the number of row tiles beside the number of CTAs.

Outputs and lse hold 7 before each call, so a row that no block writes is out of tolerance. The
tolerance is the one of ``Case.check``, and what it stands on for fp16: the reference of a half
of the softmax is the largest score of a tile that it has seen, and changes where a tile's sum
reaches 2^15. So a row's sum holds a weight of 1 (that score's own) and is at least 1, and no
weight reaches 2^15, which fp16 holds. Weights from 2^-14 up are rounded by 2^-11 of themselves,
smaller ones by 2^-25 at most: n 2^-25 max |v| over n keys, against a sum of at least 1; with
max |v| below 5 for the normal values here, 5 n 2^-25. A change of the reference scales the sums
and the roundings so far alike, and so does the joining of halves and of parts, whose weights
are at most 1 with one of them equal to 1.
"""
import numpy as np
import pytest
import torch

from paper_2608_11742_gb300 import rps
from test_gpu_prefix_attention import Case

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def uneven(n_req, nb, seed):
    """Short contexts and ten long ones at the end: the last row tiles are cut."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(1, 260, (n_req, nb))
    lens[-10:] = rng.integers(1500, 1900, (min(10, n_req), nb))
    return lens.tolist()


# (n_req, n_branch, n_q, heads, cache heads): row tiles on both sides of the CTAs of a card (152
# SMs here) and of the most that are listed by row tile (160): requests x cache heads x row tiles of a head
TILES = [(n, 1, 1, 1, 1) for n in (151, 152, 153, 155, 156, 159, 160, 161)] + [
    (5, 3, 2, 32, 32), (20, 2, 2, 16, 8), (40, 2, 3, 8, 4), (31, 1, 9, 5, 5), (53, 2, 130, 1, 1), (20, 3, 1, 56, 8)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", TILES)
def test_row_tiles_around_the_number_of_ctas(shape, dtype):
    n_req, nb, n_q, H, Hk = shape
    lens = uneven(n_req, nb, 51)
    shared = [min(x) // 2 for x in lens]
    c = Case(51, lens, shared, n_q, H, Hk, 32, dtype, causal=n_q < 9)
    c.check(*c.run())
    out = c.run(lse=False)[0]
    c.check(out, None)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("length", [200, 360, 640])
def test_like_row_tiles(length, dtype):
    """160 row tiles alike, with and without shared keys: 5 requests of 32 heads."""
    for nb, shared in ((1, None), (4, [length - 32] * 5)):
        c = Case(52, [[length] * nb] * 5, shared, 1 if nb == 1 else 16, 32, 32, 16, dtype)
        c.check(*c.run())


def test_seventeen_branches():
    """One request's base and sixteen branches, a block of 32, 32 heads: 160 row tiles."""
    c = Case(53, [[296] * 17], [264], 32, 32, 32, 16, BF16)
    c.check(*c.run())


def test_absent_sequences_among_them():
    """160 row tiles, some of absent sequences alone: their rows stay, the others are joined."""
    lens = np.array(uneven(160, 2, 54))
    lens[::7] = -1
    lens[3::11, 1] = -1
    lens[150:153] = -1
    c = Case(54, lens, None, 2, 1, 1, 16, F16)
    c.check(*c.run())


@pytest.mark.parametrize("n_req", [153, 160])
def test_replayed_with_other_lengths(n_req):
    """A captured call joins what it finds cut when it is replayed."""
    lens = np.array(uneven(n_req, 1, 55))
    c = Case(55, lens, None, 1, 1, 1, 16, BF16)
    out = torch.full_like(c.dq, 7.0)
    c.run(out, lse=False)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        c.run(out, lse=False)
    c.lens = np.minimum(lens, np.random.default_rng(56).integers(1, 1900, lens.shape))
    for at in (lens, c.lens):
        c.kv.length.copy_(torch.from_numpy(at.astype(np.int32)))
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        c.lens = at
        c.check(out, None)
