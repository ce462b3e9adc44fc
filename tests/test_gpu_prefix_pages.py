"""Attention over the paged K/V cache with page ids outside the cache in some of a sequence's many
key tiles: the rows that see a key of such a page are NaN, the others keep every bit."""
import numpy as np
import pytest
import torch

from paper_2608_11742_gb300 import rps
from test_gpu_prefix_attention import Case

pytestmark = pytest.mark.gpu


def run(c):
    """Outputs, lse and the error bits."""
    out, lse = c.run()
    return out.cpu(), lse.cpu(), rps.rps_poll_device_status()[1]


def bit_equal(a, b):
    as_int = lambda x: x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)
    return torch.equal(as_int(a), as_int(b))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("ps", [16, 32, 128, 256])
def test_bad_pages_among_many_key_tiles(ps, shared, dtype):
    """Each request of twelve has the bad pages of one of its key tiles, of every other one, or of one behind the
    limit of its first queries; each key tile has a good neighbour on both sides."""
    n_req, nb, n_q, n = 12, 2, 100, 1700
    lens = [[n - 3 * r, n - 40 - r] for r in range(n_req)]
    c = Case(61, lens, [n // 256 * 256 - 256] * n_req if shared else None, n_q, 2, 1, ps, dtype, causal=True)
    clean = run(c)
    assert clean[2] == 0 and not bool(torch.isnan(clean[0]).any())
    bad = np.zeros((n_req, nb, c.table.shape[2]), bool)  # by sequence and entry: a key of it makes a row NaN
    table = c.table.copy()
    step = max(1, 128 // ps)  # entries of a key tile
    for r in range(n_req):
        last = (lens[r][0] - 1) // ps
        entries = {0: [r * step + r % step], 1: [e for e in range(last) if e // step % 2 == 1 and e % step == 0],
                   2: [last - r % 3 if ps < 64 else last]}[r % 3]
        for e in entries:
            if e > last:
                continue
            holders = nb if shared and (e + 1) * ps <= c.d_shared[r].item() else 1  # a shared page is every sequence's
            table[r, :holders, e] = (c.k.shape[1], -1, 2 ** 31 - 1, -2 ** 31)[e % 4]
            bad[r, :holders, e] = True
    c.kv.table.copy_(torch.from_numpy(table.astype(np.int32)))
    limit = np.array(lens)[:, :, None] - n_q + np.arange(n_q) + 1  # keys that a query sees
    first = np.where(bad.any(2), bad.argmax(2) * ps, 2 ** 30)      # the first bad key of a sequence
    nan = torch.from_numpy(limit > first[:, :, None])
    assert 0 < int(nan.sum()) < nan.numel()
    for _ in range(5):
        out, lse, detail = run(c)
        assert detail == rps.DEVERR_PAGE
        assert torch.equal(torch.isnan(out).any(-1).any(-1), nan) and torch.equal(torch.isnan(out).all(-1).all(-1), nan)
        assert torch.equal(torch.isnan(lse).all(-1), nan)
        assert bit_equal(out[~nan], clean[0][~nan]) and bit_equal(lse[~nan], clean[1][~nan])
    c.kv.table.copy_(torch.from_numpy(c.table.astype(np.int32)))  # and nothing of it stays
    out, lse, detail = run(c)
    assert detail == 0 and bit_equal(out, clean[0]) and bit_equal(lse, clean[1])
