"""Pages that a caller pins by counting them once more in page_ref: no call frees, hands out or
writes them, and a compaction moves them by the rule that it states."""
import numpy as np
import pytest

from test_gpu_kvcache import Pair, i32

pytestmark = pytest.mark.gpu


def pin(p, pages, step=1):
    p.o.ref[pages] += step
    p.kv.page_ref.copy_(i32(p.o.ref))


def moved(ref, pages):
    """Where a compaction puts these pages, from the counts before it."""
    live = np.flatnonzero(ref > 0)
    n = len(live)
    place = dict(zip(live[live >= n], np.flatnonzero(ref[:n] <= 0)))
    return [int(place.get(x, x)) for x in pages]


@pytest.mark.parametrize("pages,n_req", [(60, 2), (3000, 40)])  # one block, a cluster
def test_pinned_pages_move_with_a_compaction(pages, n_req):
    p = Pair(71, 2, pages, 2, 16, n_req, 3, 8)
    n = n_req * 3
    rng = np.random.default_rng(72)
    p.resize(rng.integers(16, 8 * 16 + 1, n) if n_req > 2 else [40, 16, 70, 33, 100, 17])
    free = np.flatnonzero(p.o.ref == 0)
    held = p.o.table[n - 1, 0]  # a page of the last sequence, pinned beside it
    pins = [int(free[-1]), int(free[3]), int(held)]
    pin(p, pins)
    data = [(p.o.k[:, x].copy(), p.o.v[:, x].copy()) for x in pins]
    p.resize(np.where(np.arange(n) % 2 == 0, -1, p.o.length))  # holes below the pinned pages
    want = moved(p.o.ref, pins)
    assert want != pins
    p.compact()
    assert p.o.ref[want].min() > 0
    for x, (k, v) in zip(want, data):
        assert np.array_equal(p.o.k[:, x], k) and np.array_equal(p.o.v[:, x], v)
    p.resize(np.full(n, 100))     # takes free pages only
    p.write(0, 16)                # the row of a pinned page that a sequence holds would be left out, none is here
    p.resize(np.full(n, -1))
    assert sorted(np.flatnonzero(p.o.ref)) == sorted(want) and (p.o.ref[want] == 1).all()
    for x, (k, v) in zip(want, data):
        assert np.array_equal(p.o.k[:, x], k) and np.array_equal(p.o.v[:, x], v)
    pin(p, want, -1)
    p.compact()
    assert (p.o.ref == 0).all()


def test_a_pinned_last_page_is_copied_before_it_grows():
    p = Pair(73, 1, 12, 2, 16, 1, 2, 4)
    p.resize([20, 5])
    last = int(p.o.table[0, 1])
    pin(p, [last])
    k = p.o.k[:, last].copy()
    p.write(0, 3)                 # the pinned page's rows are left out, reported
    p.resize([25, 9])
    assert int(p.o.table[0, 1]) != last and p.o.ref[last] == 1
    p.write(0, 5)
    p.resize([-1, -1])
    assert np.array_equal(p.o.k[:, last], k) and np.flatnonzero(p.o.ref).tolist() == [last]
