"""Norms and rotation of heads (rps_rope_heads), also on the way into the paged cache
(rps_kv_append), against the oracle (oracle/drafts.py, one head at a time in fp64).

Tolerance, from the arithmetic: one rounding to the heads' type, at most e = half a step
relative (bf16 2^-8, fp16 2^-11; below fp16's normal range 2^-25 absolute), of a value whose
fp32 terms are measured by the size s = amplitude * hypot of the pair (or |y| itself):
the angle, half a turn at most, is off by 2^-32 of a turn and 2^-25 relative before and 2 ulp after the sine, 3e-7;
three roundings of the products 1.8e-7; the norm's sum of at most 256 squares takes 20
roundings of which the root halves the effect, and the reciprocal root 2 ulp: 7e-7. Together
below 2^-19 s.
"""
import numpy as np
import pytest
import torch

from oracle import drafts
from oracle import kvcache as ok
from paper_2608_11742_gb300 import rps

pytestmark = pytest.mark.gpu

E = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
EPS, AMP = 2.0 ** -20, 1.125


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def normal(rng, dtype, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype).cuda()


def make_rope(rng, D, R, dtype, norm=(True, True), interleaved=False):
    freq, _ = rps.rope_inv_freq(R, 500000.0, parts=(4.0, 8192, 32.0, 1.0)) if R else ([], 1.0)
    w = [(1.0 + 0.3 * normal(rng, torch.float32, D)).to(dtype) if n else None for n in norm]
    return rps.Rope(freq, "cuda", interleaved, AMP, w[0], w[1], EPS), freq, w


def check(got, x, w, freq, interleaved, pos, dtype, written=None):
    """got, x [..., heads, D], pos [...]."""
    g, x = got.double().cpu().numpy(), x.double().cpu().numpy()
    w = None if w is None else w.double().cpu().numpy()
    for at in np.ndindex(x.shape[:-1]):
        if written is not None and not written[at[:-1]]:
            continue
        y, size = drafts.rotate(x[at], w, EPS, freq, interleaved, AMP, int(pos[at[:-1]]))
        tol = E[dtype] * np.abs(y) + 2.0 ** -19 * size + (2.0 ** -25 if dtype == torch.float16 else 0.0) + 1e-30
        bad = ~(np.abs(g[at] - y) <= tol)
        assert not bad.any(), (at, np.abs(g[at] - y)[bad][:4], tol[bad][:4])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(128, 128), (128, 96), (128, 16), (64, 64), (64, 32), (96, 48), (96, 96), (16, 16), (256, 256),
                                 (208, 64), (128, 0), (32, 16)])
def test_parity(D, R, interleaved, dtype):
    rng = np.random.default_rng(D + R)
    rope, freq, (wq, wk) = make_rope(rng, D, R, dtype, (True, R % 32 == 0), interleaved)
    for n_seq, n_tok, H, Hk in ((1, 1, 1, 1), (2, 3, 5, 2), (1, 7, 9, 0)):
        q, pos = normal(rng, dtype, n_seq, n_tok, H, D), rng.integers(0, 2000000, (n_seq, n_tok))
        out = torch.full_like(q, 7.0)
        k = normal(rng, dtype, n_seq, n_tok, Hk, D) if Hk else None
        k_out = torch.full_like(k, 7.0) if Hk else None
        rps.rps_rope_heads(rope, q, out, k, k_out, i32(pos))
        assert rps.rps_poll_device_status()[0] == rps.RPS_OK
        check(out, q, wq, freq, interleaved, pos, dtype)
        if Hk:
            check(k_out, k, wk, freq, interleaved, pos, dtype)


def test_positions_far_out_and_without_a_list():
    """The last positions of 32 bits, negative ones, and none given (a token's index)."""
    rng = np.random.default_rng(5)
    rope, freq, (wq, _) = make_rope(rng, 128, 128, torch.bfloat16)
    far = np.array([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 16777217, 123456789]])
    q = normal(rng, torch.bfloat16, 1, 7, 3, 128)
    out = torch.empty_like(q)
    rps.rps_rope_heads(rope, q, out, pos=i32(far))
    # (in the oracle the angle is a double: 2^31 times half an ulp of the frequency, 2^-54 turns, is 2^-22 of a radian)
    check(out, q, wq, freq, False, far, torch.bfloat16)
    rps.rps_rope_heads(rope, q, out)
    check(out, q, wq, freq, False, np.arange(7)[None], torch.bfloat16)


def test_layouts_in_place_and_strides():
    """Heads before tokens, slices of a projection's rows, in place: bit for bit as contiguous rows."""
    rng = np.random.default_rng(6)
    rope, _, _ = make_rope(rng, 128, 64, torch.bfloat16)
    q, k, pos = normal(rng, torch.bfloat16, 2, 37, 6, 128), normal(rng, torch.bfloat16, 2, 37, 2, 128), i32(rng.integers(0, 9999, (2, 37)))
    a, b = torch.empty_like(q), torch.empty_like(k)
    rps.rps_rope_heads(rope, q, a, k, b, pos)
    rows = torch.full((2, 37, 11, 144), 7.0, dtype=torch.bfloat16, device="cuda")
    rows[:, :, 1:7, :128], rows[:, :, 7:9, :128] = q, k
    qs, ks = rows[:, :, 1:7, :128], rows[:, :, 7:9, :128]
    by_head = torch.full((2, 6, 37, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    rps.rps_rope_heads(rope, qs, by_head.transpose(1, 2), ks, ks, pos)
    assert torch.equal(by_head.transpose(1, 2), a) and torch.equal(ks, b) and torch.equal(qs, q)
    rest = rows.clone()
    rest[:, :, 1:9, :128] = 7.0
    assert bool((rest == 7.0).all())
    rps.rps_rope_heads(rope, q, q, pos=pos)
    assert torch.equal(q, a)


def test_many_rows_as_few():
    """More tasks than fit the card at once, four passes a task: bit for bit as calls of one token, which take one."""
    rng = np.random.default_rng(7)
    rope, _, _ = make_rope(rng, 128, 128, torch.float16)
    q, k, pos = normal(rng, torch.float16, 1, 2000, 28, 128), normal(rng, torch.float16, 1, 2000, 4, 128), i32(rng.integers(0, 10 ** 6, (1, 2000)))
    a, b = torch.empty_like(q), torch.empty_like(k)
    rps.rps_rope_heads(rope, q, a, k, b, pos)
    for t in (0, 1, 999, 1999):
        x, y = q[:, t:t + 1].clone(), k[:, t:t + 1].clone()
        rps.rps_rope_heads(rope, x, x, y, y, pos[:, t:t + 1].contiguous())
        assert torch.equal(x, a[:, t:t + 1]) and torch.equal(y, b[:, t:t + 1])


def test_values_that_are_not_finite_stay_in_their_heads():
    rng = np.random.default_rng(8)
    rope, freq, (wq, _) = make_rope(rng, 128, 128, torch.bfloat16)
    q = normal(rng, torch.bfloat16, 1, 4, 8, 128)
    clean = torch.empty_like(q)
    rps.rps_rope_heads(rope, q, clean)
    q[0, 1, 3, 5], q[0, 2, 6, 100] = float("nan"), float("inf")
    q[0, 3, 0] = 0.0
    out = torch.empty_like(q)
    rps.rps_rope_heads(rope, q, out)
    same = torch.ones((4, 8), dtype=torch.bool)
    same[1, 3] = same[2, 6] = same[3, 0] = False
    assert torch.equal(out[0][same.cuda()], clean[0][same.cuda()])
    assert bool(torch.isnan(out[0, 1, 3]).all()) and bool((out[0, 3, 0] == 0).all())


class Append:
    def __init__(self, seed, lens, H, Hk, ps, n_new, dtype=torch.bfloat16, tokens_first=False, R=128, interleaved=False, layers=2):
        rng = self.rng = np.random.default_rng(seed)
        lens = np.array(lens)
        n_req, nb = lens.shape
        pages = lambda n: 0 if n <= 0 else -(-int(n) // ps)
        width = max(1, max(pages(n) for n in lens.ravel()))
        n_pages = sum(pages(n) for n in lens.ravel()) + 3
        place, at = rng.permutation(n_pages), 0
        table = np.full((n_req, nb, width), -1)
        for r, b in np.ndindex(n_req, nb):
            m = pages(lens[r, b])
            table[r, b, :m] = place[at:at + m]
            at += m
        ref = np.bincount(table[table >= 0].ravel(), minlength=n_pages)
        k = normal(rng, dtype, layers, n_pages, Hk, ps, 128)
        v = normal(rng, dtype, layers, n_pages, Hk, ps, 128)
        if tokens_first:
            k, v = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (k, v))
        self.kv = rps.KvCacheBuf(k, v, i32(ref), i32(table), i32(lens))
        self.o = ok.Cache(ref, table.reshape(-1, width), lens.ravel(), ps, k.double().cpu().numpy(), v.double().cpu().numpy())
        self.rows = normal(rng, dtype, n_req, nb, n_new, H + 2 * Hk, 128)
        self.q, self.kn, self.vn = self.rows[..., :H, :], self.rows[..., H:H + Hk, :], self.rows[..., H + Hk:, :]
        self.rope, self.freq, (self.wq, self.wk) = make_rope(rng, 128, R, dtype, (True, True), interleaved)
        self.interleaved, self.dtype, self.n_new, self.lens = interleaved, dtype, n_new, lens

    def check(self, layer=1, count=None, pos=None, status=0):
        n_seq = self.kv.n_seq
        before_k, before_v = self.kv.k.clone(), self.kv.v.clone()
        out = torch.full(self.q.shape, 7.0, dtype=self.dtype, device="cuda")
        rps.rps_kv_append(self.kv, layer, self.rope, self.kn, self.vn, self.q, out, None if count is None else i32(count),
                          None if pos is None else i32(pos))
        bits = rps.rps_poll_device_status()[1]
        assert bits == status, hex(bits)
        flat = lambda x: x.reshape(n_seq, *x.shape[2:])
        got_q, q, kn, vn = flat(out), flat(self.q), flat(self.kn), flat(self.vn)
        written, where = np.zeros((n_seq, self.n_new), bool), np.zeros((n_seq, self.n_new), np.int64)
        want_k, want_v = before_k.clone(), before_v.clone()
        rows = []
        for s, i, p, page in drafts.append_places(self.o, self.n_new, count):
            written[s, i], where[s, i] = True, p if pos is None else np.asarray(pos).reshape(n_seq, -1)[s, i]
            if page is not None:
                rows.append((s, i, page, p % self.o.ps))
                want_v[layer, page, :, p % self.o.ps] = vn[s, i]
        assert self.o.err == status
        check(got_q, q, self.wq, self.freq, self.interleaved, where, self.dtype, written)
        assert bool((got_q[torch.from_numpy(~written).cuda()] == 7.0).all())
        assert torch.equal(self.kv.v, want_v)
        for s, i, page, row in rows:
            check(self.kv.k[layer, page, :, row][None], kn[s, i][None], self.wk, self.freq, self.interleaved, where[s, i][None], self.dtype)
            want_k[layer, page, :, row] = self.kv.k[layer, page, :, row]
        assert torch.equal(self.kv.k, want_k), "other rows of the cache were written"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ps", [16, 64, 256])
def test_append(ps, dtype):
    lens = [[1, 40, -1, 0], [ps, ps + 1, 300, 7]]
    for n_new, interleaved, R, first in ((1, False, 128, False), (5, True, 64, True), (17, False, 96, False)):
        Append(ps + n_new, lens, 6, 2, ps, n_new, dtype, first, R, interleaved).check()


def test_append_of_ragged_counts_at_given_positions():
    a = Append(30, [[60, 33, 20], [90, -1, 4]], 4, 4, 16, 9)
    a.check(count=[9, 0, 3, 12, 5, 9], pos=a.rng.integers(-5, 70000, (2, 3, 9)))


def test_append_of_one_branch_and_of_plain_rows():
    a = Append(31, [[60], [33], [20]], 4, 4, 16, 3)
    a.check()
    # no rope: rows as they are, as rps_kv_write has them
    b, c = Append(32, [[60], [33], [20]], 4, 4, 16, 3), Append(32, [[60], [33], [20]], 4, 4, 16, 3)
    rps.rps_kv_append(b.kv, 0, None, b.kn, b.vn)
    rps.rps_kv_write(c.kv, 0, c.kn.contiguous(), c.vn.contiguous())
    assert torch.equal(b.kv.k, c.kv.k) and torch.equal(b.kv.v, c.kv.v) and rps.rps_poll_device_status()[0] == rps.RPS_OK


def test_append_leaves_out_shared_and_bad_pages():
    a = Append(33, [[60, 33, 20]], 4, 2, 16, 20)
    shared, gone = int(a.o.table[0, 3]), int(a.o.table[1, 1])
    a.kv.page_ref[shared] += 1
    a.o.ref[shared] += 1
    a.kv.table[0, 1, 1] = a.kv.k.shape[1]
    a.o.table[1, 1] = a.kv.k.shape[1]
    a.check(status=rps.DEVERR_SHARED | rps.DEVERR_PAGE)
    assert gone >= 0


def test_append_of_a_length_beyond_the_table():
    a = Append(34, [[30, 16]], 2, 2, 16, 4)
    a.kv.length[0, 0] = 1000
    a.o.length[0] = 1000
    a.check(status=rps.DEVERR_PAGE)


def test_offsets_beyond_32_bits():
    """A cache beyond 2^32 bytes, and rows beyond 2^31 elements."""
    rng = np.random.default_rng(35)
    kv = rps.KvCacheBuf.alloc(2, 20000, 8, 64, 1, 1, 2, "cuda")
    kv.table.copy_(i32([[[19999, 17]]]))
    kv.length.fill_(70)
    kv.page_ref[19999] = kv.page_ref[17] = 1
    rope, freq, (wq, wk) = make_rope(rng, 128, 128, torch.bfloat16)
    k, v = normal(rng, torch.bfloat16, 1, 1, 70, 8, 128), normal(rng, torch.bfloat16, 1, 1, 70, 8, 128)
    rps.rps_kv_append(kv, 1, rope, k, v)
    got = torch.cat([kv.k[1, 19999].transpose(0, 1), kv.k[1, 17, :, :6].transpose(0, 1)])
    check(got[60:], k[0, 0, 60:], wk, freq, False, np.arange(60, 70), torch.bfloat16)
    assert torch.equal(torch.cat([kv.v[1, 19999].transpose(0, 1), kv.v[1, 17, :, :6].transpose(0, 1)]), v[0, 0])
    q = torch.zeros((3, 300000, 20, 128), dtype=torch.bfloat16, device="cuda")  # 2.3 G elements
    q[2, -1] = normal(rng, torch.bfloat16, 20, 128)
    x, pos = q[2:, -1:].clone(), i32(np.full((3, 300000), 12345))
    rps.rps_rope_heads(rope, q, q, pos=pos)
    check(q[2:, -1:], x, wq, freq, False, np.full((1, 1), 12345), torch.bfloat16)
    assert bool((q[0, 0] == 0).all()) and rps.rps_poll_device_status()[0] == rps.RPS_OK


def test_on_a_side_stream_and_from_a_graph():
    a = Append(36, [[60, 33], [20, 90]], 4, 2, 16, 3)
    out, first = torch.zeros_like(a.q), torch.zeros_like(a.q)
    run = lambda to, stream=None: rps.rps_kv_append(a.kv, 0, a.rope, a.kn, a.vn, a.q, to, stream=stream)
    run(first)
    k = a.kv.k.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run(out, side)
    side.synchronize()
    assert torch.equal(out, first) and torch.equal(a.kv.k, k)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        run(out)
    out.zero_()
    a.kv.k.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first) and int((a.kv.k != 0).sum()) > 0


def any_bits(rng, dtype, *shape):
    """Every kind of 16-bit pattern: zeros of both signs, the smallest, infinities, NaN with their payloads."""
    x = rng.integers(-2 ** 15, 2 ** 15, shape).astype(np.int16)
    x.reshape(-1)[::5] = rng.choice(np.array([0, -2 ** 15, 1, 0x7f80, -0x80, 0x7c00, -0x400, 0x7fff, 0x7f81], np.int16), x.reshape(-1)[::5].size)
    return torch.from_numpy(x).cuda().view(dtype)


def bits(x):
    return x.contiguous().view(torch.int16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(128, 96), (128, 16), (128, 0), (64, 16), (16, 0), (96, 48), (256, 208), (208, 64)])
def test_elements_that_are_not_rotated_stay_as_they_are(D, R, interleaved, dtype):
    """A side without norm: bit for bit past the rotated elements, whatever they hold, which also changes no rotated one."""
    rng = np.random.default_rng(39)
    rope, _, _ = make_rope(rng, D, R, dtype, (False, False), interleaved)
    for heads in (1, 5, 40):
        q, k, pos = normal(rng, dtype, 2, 3, heads, D), normal(rng, dtype, 2, 3, 2, D), i32(rng.integers(0, 9999, (2, 3)))
        clean = torch.empty_like(q)
        rps.rps_rope_heads(rope, q, clean, pos=pos)
        q[..., R:], k[..., R:] = any_bits(rng, dtype, 2, 3, heads, D - R), any_bits(rng, dtype, 2, 3, 2, D - R)
        out, k_out = torch.empty_like(q), torch.empty_like(k)
        rps.rps_rope_heads(rope, q, out, k, k_out, pos)
        assert torch.equal(bits(out[..., R:]), bits(q[..., R:])) and torch.equal(bits(k_out[..., R:]), bits(k[..., R:]))
        assert torch.equal(bits(out[..., :R]), bits(clean[..., :R]))
        # the other side's norm is no matter
        half, _, (wq, _) = make_rope(rng, D, R, dtype, (True, False), interleaved)
        rps.rps_rope_heads(half, clean, out, k, k_out, pos)
        assert torch.equal(bits(k_out[..., R:]), bits(k[..., R:]))
        check(out, clean, wq, half._made_of[0], interleaved, pos.cpu().numpy(), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [0, 16, 64, 112])
def test_normed_elements_that_are_not_rotated_take_nothing_from_others(R, interleaved, dtype):
    """With a norm an infinity is NaN and the finite elements are zeros, by the formula x w / inf; zeros keep their signs."""
    rng = np.random.default_rng(40)
    D = 128
    rope, _, (w, _) = make_rope(rng, D, R, dtype, (True, True), interleaved)
    assert bool((w > 0).any()) and bool(torch.isfinite(w).all())
    for at in (R, R + 1, R + 8, (R + D) // 2, D - 1):
        q = normal(rng, dtype, 1, 2, 5, D)
        q[0, 0, 1, at], q[0, 1, 3, at] = float("inf"), -float("inf")
        q[0, 0, 2, at] = -0.0
        out = torch.empty_like(q)
        rps.rps_rope_heads(rope, q, out)
        assert bool(torch.isnan(out[0, 0, 1, at])) and bool(torch.isnan(out[0, 1, 3, at]))
        rest = [i for i in range(D) if i != at]
        assert bool((out[0, 0, 1, rest] == 0).all()) and bool((out[0, 1, 3, rest] == 0).all())
        assert bool(out[0, 0, 2, at] == 0) and bool(torch.signbit(out[0, 0, 2, at]) != torch.signbit(w[at]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R", [None, 0, 64])
def test_append_of_rows_that_hold_anything(R, dtype):
    """Without rotation and norm, keys, values and queries bit for bit, as rps_kv_write has them; with R, past it."""
    rng = np.random.default_rng(41)
    a, b = (Append(42, [[60, 33], [20, 90]], 6, 2, 16, 7, dtype) for _ in range(2))
    rope = None if R is None else make_rope(rng, 128, R, dtype, (False, False))[0]
    r = R or 0
    a.rows[..., r:] = any_bits(rng, dtype, *a.rows.shape[:-1], 128 - r)
    out = torch.empty_like(a.q)
    rps.rps_kv_append(a.kv, 1, rope, a.kn, a.vn, a.q, out)
    rps.rps_kv_write(b.kv, 1, a.kn.contiguous(), a.vn.contiguous())
    assert rps.rps_poll_device_status()[0] == rps.RPS_OK
    assert torch.equal(bits(out[..., r:]), bits(a.q[..., r:]))
    assert torch.equal(bits(a.kv.k[..., r:]), bits(b.kv.k[..., r:])) and torch.equal(bits(a.kv.v), bits(b.kv.v))


def test_refusals_of_the_binding():
    rng = np.random.default_rng(37)
    bf16 = torch.bfloat16
    rope, _, _ = make_rope(rng, 128, 64, bf16)
    q = normal(rng, bf16, 2, 3, 4, 128)
    for kw, err in ((dict(q=q.cpu()), ValueError), (dict(q=q.float()), ValueError), (dict(q_out=q.half()), TypeError),
                    (dict(q_out=q[:, :2]), ValueError), (dict(q=q[..., :64]), ValueError), (dict(k=q), ValueError),
                    (dict(k=q[:, :2], k_out=q[:, :2]), ValueError), (dict(pos=i32([1, 2])), ValueError),
                    (dict(pos=torch.zeros((2, 3), device="cuda")), ValueError), (dict(q=q.transpose(2, 3)), ValueError),
                    (dict(q=q.half(), q_out=q.half()), ValueError)):
        with pytest.raises(err):
            rps.rps_rope_heads(**{**dict(rope=rope, q=q, q_out=torch.empty_like(q)), **kw})
    with pytest.raises(ValueError):
        rps.Rope([1.0], "cuda", q_weight=torch.ones(128, device="cuda"))
    a = Append(38, [[60, 33], [20, 90]], 4, 2, 16, 3)
    for kw, err in ((dict(k_new=a.kn[:, :1]), ValueError), (dict(v_new=a.vn[:, :, :2]), ValueError), (dict(k_new=a.kn.half()), TypeError),
                    (dict(q=a.q), ValueError), (dict(q=a.q, q_out=a.q[:, :, :2]), ValueError), (dict(n_tok=i32([1])), ValueError),
                    (dict(pos=i32([1])), ValueError), (dict(layer=2), rps.RPSError), (dict(k_new=a.kn.cpu()), ValueError),
                    (dict(k_new=a.kn.transpose(0, 1), v_new=a.vn.transpose(0, 1)), ValueError)):
        with pytest.raises(err):
            rps.rps_kv_append(**{**dict(kv=a.kv, layer=0, rope=a.rope, k_new=a.kn, v_new=a.vn), **kw})
