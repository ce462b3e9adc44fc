"""Operators of a layer's attention block over the paged K/V cache, each in its plain form and as the package's calls.

Five kinds of passes:

* ``rope``: the norms of queries and keys for each head and the rotation by their
  positions (``rps.rps_rope_heads``), as a forward pass without a cache needs them;
* ``append``: the same on the way into the paged cache, values with them
  (``rps.rps_kv_append``);
* ``masks``: the ancestors and the positions of drafted tokens from their parents
  (``rps.rps_tree_masks``);
* ``tree``: attention of a sequence's newest tokens over its cache, drafted tokens
  seeing their own ancestors (``rps.rps_tree_attention_fwd``); without a mask the
  newest tokens are a chain, of one token in ordinary decoding;
* ``keep``: the keys and values of the accepted path move to the front of the
  drafted tokens (``rps.rps_kv_keep_path``).

``own`` selects the package's calls; otherwise ``run`` computes the same in
elementary torch operations, in 32 bits, angles in 64.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
# No case costs more than the largest listed ones.
MAX_FLOPS = 80e9
MAX_CACHE_BYTES = 1.5e9
MAX_ROW_BYTES = 0.7e9


def _rope(name, n_seq, n_tok, H, Hk, D, R, interleaved, norm, far, dtype):
    """R: rotated elements of a head; far: the largest position."""
    c = dict(kind="rope", n_seq=n_seq, n_tok=n_tok, H=H, Hk=Hk, D=D, R=R, interleaved=interleaved, norm=norm, far=far, dtype=dtype)
    return dict(name=name, **c) if name else c


def _append(name, n_seq, n_new, H, Hk, ps, length, R, interleaved, norm, ragged, dtype):
    """length: range of the sequences' tokens, the new ones among them; ragged: sequences bring fewer than n_new."""
    c = dict(kind="append", n_seq=n_seq, n_new=n_new, H=H, Hk=Hk, ps=ps, len_lo=length[0], len_hi=length[1], D=128, R=R,
             interleaved=interleaved, norm=norm, ragged=ragged, dtype=dtype)
    return dict(name=name, **c) if name else c


def _masks(name, n_seq, n_tok, fan, ragged):
    """fan: children of a token, about."""
    c = dict(kind="masks", n_seq=n_seq, n_tok=n_tok, fan=fan, ragged=ragged)
    return dict(name=name, **c) if name else c


def _tree(name, n_seq, n_q, H, Hk, ps, ctx, tree, ragged, dtype):
    """ctx: range of the tokens before the drafted ones; tree: drafted tokens have parents, else they are a chain."""
    c = dict(kind="tree", n_seq=n_seq, n_q=n_q, H=H, Hk=Hk, ps=ps, ctx_lo=ctx[0], ctx_hi=ctx[1], D=128, tree=tree,
             ragged=ragged, dtype=dtype)
    return dict(name=name, **c) if name else c


def _keep(name, n_seq, n_q, n_keep, layers, Hk, ps, ctx, dtype):
    c = dict(kind="keep", n_seq=n_seq, n_q=n_q, n_keep=n_keep, layers=layers, Hk=Hk, ps=ps, ctx_lo=ctx[0], ctx_hi=ctx[1],
             D=128, dtype=dtype)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token each of a few users: latency
        _rope("rope-token", 4, 1, 28, 4, 128, 128, False, True, 30000, "bf16"),
        # a long prompt far into its positions, three quarters of each head rotated, pairs side by side
        _rope("rope-prompt", 2, 8111, 32, 32, 128, 96, True, False, 1000000, "f16"),
        # ordinary decoding of a batch: one token a sequence into its page, its query rotated in the same call
        _append("append-token", 64, 1, 28, 4, 16, (1, 4000), 128, False, True, False, "bf16"),
        # the blocks of a batch's branches
        _append("append-serve", 576, 32, 32, 32, 16, (40, 130), 128, False, True, True, "bf16"),
        # one user's drafted tokens
        _masks("masks-one", 1, 32, 3, False),
        # a batch of deep ones, of odd sizes
        _masks("masks-serve", 500, 253, 2, True),
        # one user's drafted tokens over a short context: latency
        _tree("tree-one", 1, 16, 32, 32, 16, (328, 328), True, False, "bf16"),
        # token by token generation of many users, contexts ragged
        _tree("tree-token", 64, 1, 28, 4, 16, (200, 8000), False, False, "bf16"),
        # drafted trees of a batch, numbers of tokens ragged, two row tiles of query rows
        _tree("tree-serve", 64, 32, 32, 4, 64, (500, 4000), True, True, "bf16"),
        # large trees over long contexts, fp16
        _tree("tree-long", 2, 64, 32, 8, 64, (24000, 32700), True, False, "f16"),
        # one user's accepted path, four layers
        _keep("keep-one", 1, 32, 5, 4, 8, 16, (328, 328), "bf16"),
        # a batch's paths, whole stack of layers
        _keep("keep-serve", 64, 64, 17, 32, 8, 16, (100, 160), "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "masks", "tree", "tree", "tree", "keep"])
    while True:
        dtype = rng.choice(["bf16", "bf16", "f16"])
        Hk, ps = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([16, 16, 32, 64, 128, 256])
        H = Hk * rng.choice([1, 1, 2, 4, 7, 8, 16])
        norm, interleaved = rng.choice([True, True, False]), rng.choice([True, False])
        if kind == "rope":
            D = rng.choice([64, 96, 128, 128, 256])
            c = _rope(None, _log_int(rng, 1, 64), _log_int(rng, 1, 16000), H, Hk, D, rng.choice([16, 32, 64, D, D]), interleaved,
                      norm, _log_int(rng, 100, 1000000), dtype)
            if H <= 64 and work(c)["bytes"] <= MAX_ROW_BYTES:
                return c
        elif kind == "append":
            n_new = rng.choice([1, 1, _log_int(rng, 2, 64)])
            hi = n_new + _log_int(rng, 1, 4000)
            c = _append(None, _log_int(rng, 1, 600), n_new, H, Hk, ps, (n_new, hi), rng.choice([32, 64, 128, 128]), interleaved,
                        norm, rng.choice([True, False]), dtype)
            if H <= 64 and work(c)["bytes"] <= MAX_ROW_BYTES and c["n_seq"] * (hi // ps + 1) * ps * Hk * 512 <= MAX_CACHE_BYTES:
                return c
        elif kind == "masks":
            return _masks(None, _log_int(rng, 1, 500), _log_int(rng, 1, 253), rng.choice([1, 2, 3, 4, 8]), rng.choice([True, False]))
        elif kind == "tree":
            n_q = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
            hi = _log_int(rng, 16, 130000)
            c = _tree(None, _log_int(rng, 1, 256), n_q, H, Hk, ps, (rng.choice([hi, max(1, hi // 8)]), hi),
                      rng.choice([True, True, False]), rng.choice([True, False]), dtype)
            keys = c["n_seq"] * (hi + n_q + ps)
            if H <= 64 and work(c)["flops"] <= MAX_FLOPS and keys * Hk * 512 <= MAX_CACHE_BYTES and keys * n_q * H * 4 <= 3e9:
                return c
        else:
            n_q = _log_int(rng, 2, 64)
            hi = _log_int(rng, 1, 2000)
            c = _keep(None, _log_int(rng, 1, 256), n_q, rng.randint(1, max(1, n_q // 2)), rng.choice([1, 2, 4, 16, 32]), Hk, ps,
                      (max(1, hi // 4), hi), dtype)
            if c["n_seq"] * ((hi + n_q) // ps + 1) * ps * c["layers"] * Hk * 512 <= MAX_CACHE_BYTES:
                return c


# ---------------------------------------------------------------- inputs
def _dt(case):
    return torch.float16 if case.get("dtype") == "f16" else torch.bfloat16


def _normal(shape, dtype, g):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _inv_freq(R):
    """Radians per position of each pair: base 500000, the slow half of them stretched by four (a scaled context)."""
    f = 500000.0 ** -(np.arange(0, R, 2) / R)
    f[R // 4:] /= 4.0
    return f


AMPLITUDE = 1.125  # of the rotated elements, as scaled contexts have it


def _parents(rs, n_seq, n_tok, fan):
    """Drafted tokens in the order of their depth, about; a parent comes before its children, -1: the context's end."""
    i = np.arange(n_tok)
    p = i // fan - 1 + rs.integers(0, 2, (n_seq, n_tok))
    return np.minimum(p, i - 1)


def _ancestors(parent):
    """[n_seq][n_tok][n_tok]: whether token i sees drafted token j; and the depths."""
    n_seq, n = parent.shape
    sees, depth = np.zeros((n_seq, n, n), bool), np.zeros((n_seq, n), np.int64)
    for i in range(n):
        p = parent[:, i]
        here = p >= 0
        sees[here, i] = sees[here, p[here]]
        depth[here, i] = depth[here, p[here]] + 1
        sees[:, i, i] = True
    return sees, depth


def _words(sees):
    """The same as words of 32 bits, bit j % 32 of word j // 32."""
    n_seq, n, _ = sees.shape
    wide = np.zeros((n_seq, n, -(-n // 32) * 32), np.uint64)
    wide[:, :, :n] = sees
    bit = np.uint64(1) << np.arange(32, dtype=np.uint64)
    return (wide.reshape(n_seq, n, -1, 32) * bit).sum(-1).astype(np.uint32).view(np.int32)


def _book(rs, length, width, ps, spare=3):
    """Page tables in a shuffled cache with room for every sequence's largest length, as [n_seq][width]; its pages."""
    used = np.arange(width) < (-(-length // ps))[:, None]
    table = np.full((len(length), width), -1, np.int64)
    n_pages = len(length) * width + spare
    table[used] = rs.permutation(n_pages)[: int(used.sum())]
    return table, n_pages


def _norm_weights(case, g):
    if not case["norm"]:
        return None, None
    return [(1.0 + 0.2 * _normal((case["D"],), torch.float32, g)).to(_dt(case)) for _ in range(2)]


def _counts(case, rs, most):
    """Tokens that each sequence brings."""
    lo = 1 if case["ragged"] else most
    return rs.integers(lo, most + 1, case["n_seq"])


def _tree_inputs(case, seed):
    rs = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n_seq, n_q, Hk, ps, D = case["n_seq"], case["n_q"], case["Hk"], case["ps"], case["D"]
    count = _counts(case, rs, n_q)
    ctx = rs.integers(case["ctx_lo"], case["ctx_hi"] + 1, n_seq)
    width = -(-(case["ctx_hi"] + n_q) // ps)
    table, n_pages = _book(rs, ctx + count, width, ps)
    sees, _ = _ancestors(_parents(rs, n_seq, n_q, 3)) if case["tree"] else (np.tril(np.ones((1, n_q, n_q), bool)), None)
    k, v = (_normal((1, n_pages, Hk, ps, D), _dt(case), g) for _ in range(2))
    q = _normal((n_seq, 1, n_q, case["H"], D), _dt(case), g)
    q *= 2.0  # scores of about 2 nats' spread
    return q, k, v, count, ctx, table, sees


def _append_inputs(case, seed):
    rs = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, n_new, Hk, ps, D = case["n_seq"], case["n_new"], case["Hk"], case["ps"], case["D"]
    count = _counts(case, rs, n_new)
    length = rs.integers(case["len_lo"], case["len_hi"] + 1, n)
    table, n_pages = _book(rs, length, -(-case["len_hi"] // ps), ps)
    k, v = (_normal((1, n_pages, Hk, ps, D), _dt(case), g) for _ in range(2))
    # queries, keys and values as one projection leaves them
    rows = _normal((n, 1, n_new, case["H"] + 2 * Hk, D), _dt(case), g)
    return rows, k, v, count, length, table, _norm_weights(case, g)


def _rope_inputs(case, seed):
    rs = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, n_tok, D = case["n_seq"], case["n_tok"], case["D"]
    pos = rs.integers(0, max(1, case["far"] - n_tok) + 1, (n, 1)) + np.arange(n_tok)
    rows = _normal((n, n_tok, case["H"] + case["Hk"], D), _dt(case), g)
    return rows, pos, _norm_weights(case, g)


def _keep_inputs(case, seed):
    """Paths whose moved rows are not read again by a second pass: entries in their place, or behind the kept ones."""
    rs = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, n_q, m, ps = case["n_seq"], case["n_q"], case["n_keep"], case["ps"]
    ctx = rs.integers(case["ctx_lo"], case["ctx_hi"] + 1, n)
    table, n_pages = _book(rs, ctx + n_q, -(-(case["ctx_hi"] + n_q) // ps), ps)
    path, keep = np.zeros((n, m), np.int64), rs.integers(1, m + 1, n)
    for s in range(n):
        still = int(rs.integers(0, min(2, keep[s]) + 1))
        path[s, :still] = np.arange(still)
        later = np.arange(keep[s], n_q)
        take = min(len(later), int(keep[s]) - still)
        keep[s] = still + take
        path[s, still:keep[s]] = np.sort(rs.choice(later, take, replace=False))
    shape = (case["layers"], n_pages, case["Hk"], ps, case["D"])
    return _normal(shape, _dt(case), g), _normal(shape, _dt(case), g), ctx, table, path, keep


def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case}
    if kind == "rope":
        rows, pos, (s["wq"], s["wk"]) = _rope_inputs(case, seed)
        H = case["H"]
        s["q"], s["k"], s["pos"] = rows[:, :, :H], rows[:, :, H:], _i32(pos)
        s["q_out"], s["k_out"] = torch.empty(s["q"].shape, dtype=_dt(case), device="cuda"), torch.empty(s["k"].shape, dtype=_dt(case), device="cuda")
    elif kind == "append":
        rows, s["k"], s["v"], count, length, table, (s["wq"], s["wk"]) = _append_inputs(case, seed)
        H, Hk = case["H"], case["Hk"]
        s["q"], s["k_new"], s["v_new"] = rows[:, :, :, :H], rows[:, :, :, H:H + Hk], rows[:, :, :, H + Hk:]
        s["q_out"] = torch.zeros(s["q"].shape, dtype=_dt(case), device="cuda")
        s["count"] = _i32(count) if case["ragged"] else None
        s["table"], s["len"] = _i32(table[:, None]), _i32(length[:, None])
    elif kind == "masks":
        rs = np.random.default_rng(seed)
        s["parent"] = _i32(_parents(rs, case["n_seq"], case["n_tok"], case["fan"]))
        count = _counts(case, rs, case["n_tok"])
        s["count"], s["len"] = _i32(count), _i32(count + rs.integers(0, 5000, case["n_seq"]))
        s["mask"] = torch.zeros((case["n_seq"], case["n_tok"], -(-case["n_tok"] // 32)), dtype=torch.int32, device="cuda")
        s["pos"] = torch.zeros_like(s["parent"])
    elif kind == "tree":
        s["q"], s["k"], s["v"], count, ctx, table, sees = _tree_inputs(case, seed)
        s["count"] = _i32(count) if case["ragged"] else None
        s["table"], s["len"] = _i32(table[:, None]), _i32((ctx + count)[:, None])
        s["mask"] = _i32(_words(sees)) if case["tree"] else None
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(s["q"].shape[:4], dtype=torch.float32, device="cuda")
    else:
        s["k"], s["v"], ctx, table, path, keep = _keep_inputs(case, seed)
        s["table"], s["len"] = _i32(table[:, None]), _i32((ctx + case["n_q"])[:, None])
        s["path"], s["keep"] = _i32(path), _i32(keep)
        s["new_len"] = torch.zeros_like(s["len"])
    if "R" in case:
        s["inv_freq"] = torch.from_numpy(_inv_freq(case["R"])).cuda()
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_2608_11742_gb300 import rps

    case = s["case"]
    if "R" in case:
        s["rope"] = rps.Rope(_inv_freq(case["R"]), "cuda", interleaved=case["interleaved"], amplitude=AMPLITUDE,
                             q_weight=s["wq"], k_weight=s["wk"], eps=EPS)
    if "table" in s:
        ref = torch.zeros(s["k"].shape[1], dtype=torch.int32, device="cuda")
        ref[s["table"][s["table"] >= 0].long()] = 1
        s["kv"] = rps.KvCacheBuf(s["k"], s["v"], ref, s["table"], s["len"])
    if case["kind"] == "tree":
        n = rps.rps_tree_attention_workspace_bytes(s["kv"], case["n_q"], case["H"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------- the package's calls
def _run_own(s):
    from paper_2608_11742_gb300 import rps

    kind = s["case"]["kind"]
    if kind == "rope":
        rps.rps_rope_heads(s["rope"], s["q"], s["q_out"], s["k"], s["k_out"], s["pos"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "append":
        rps.rps_kv_append(s["kv"], 0, s["rope"], s["k_new"], s["v_new"], s["q"], s["q_out"], n_tok=s["count"])
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if kind == "masks":
        rps.rps_tree_masks(s["parent"], s["mask"], s["pos"], n_tok=s["count"], length=s["len"])
        return {"mask": s["mask"], "pos": s["pos"]}
    if kind == "tree":
        rps.rps_tree_attention_fwd(s["q"], s["kv"], 0, s["out"], s["ws"], s["mask"], s["case"]["D"] ** -0.5, n_tok=s["count"],
                                   lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    rps.rps_kv_keep_path(s["kv"], s["path"], s["keep"], s["new_len"], s["case"]["n_q"])
    return {"k": s["k"], "v": s["v"], "new_len": s["new_len"]}


# ---------------------------------------------------------------- the plain forms
def _plain_rotate(s, x, w, pos):
    """x [..., heads, D] with positions [...]: norm, rotation, one rounding."""
    case = s["case"]
    R = case["R"]
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt(y.pow(2).mean(-1, keepdim=True) + EPS) * w.float()
    a = pos.double()[..., None, None] * s["inv_freq"]
    cos, sin = (torch.cos(a) * AMPLITUDE).float(), (torch.sin(a) * AMPLITUDE).float()
    z = y.clone()
    first, second = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
    z[..., first] = y[..., first] * cos - y[..., second] * sin
    z[..., second] = y[..., second] * cos + y[..., first] * sin
    return z.to(x.dtype)


def _plain_append(s):
    case = s["case"]
    n, n_new, ps = case["n_seq"], case["n_new"], case["ps"]
    i = torch.arange(n_new, device="cuda")
    count = s["count"].long() if case["ragged"] else torch.full((n,), n_new, device="cuda")
    pos = s["len"].long() - count[:, None] + i
    there = (i < count[:, None]) & (pos >= 0)
    q, k = (_plain_rotate(s, x[:, 0], w, pos) for x, w in ((s["q"], s["wq"]), (s["k_new"], s["wk"])))
    s["q_out"][:, 0] = torch.where(there[..., None, None], q, s["q_out"][:, 0])
    at = pos.clamp(0, s["table"].shape[2] * ps - 1)
    page = torch.gather(s["table"][:, 0].long(), 1, at // ps)[there]
    row = (at % ps)[there]
    s["k"][0][page, :, row] = k[there]
    s["v"][0][page, :, row] = s["v_new"][:, 0][there]
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _plain_masks(s):
    """Ancestors by doubling: who is seen within 2^r steps, r up to the depth's logarithm."""
    case = s["case"]
    n = case["n_tok"]
    i = torch.arange(n, device="cuda")
    there = i < s["count"][:, None]
    step = torch.where(s["parent"][:, :, None] == i, 1.0, 0.0)
    sees = step + torch.eye(n, device="cuda")
    # eight squarings reach 256 steps
    sees = torch.matmul(sees, sees).clamp(max=1.0)
    sees = torch.matmul(sees, sees).clamp(max=1.0)
    sees = torch.matmul(sees, sees).clamp(max=1.0)
    sees = torch.matmul(sees, sees).clamp(max=1.0)
    sees = torch.matmul(sees, sees).clamp(max=1.0)
    sees = torch.matmul(sees, sees).clamp(max=1.0)
    sees = torch.matmul(sees, sees).clamp(max=1.0)
    sees = torch.matmul(sees, sees).clamp(max=1.0)
    words = s["mask"].shape[2]
    wide = torch.zeros((case["n_seq"], n, 32 * words), dtype=torch.int64, device="cuda")
    wide[:, :, :n] = sees.long()
    bits = (wide.view(case["n_seq"], n, words, 32) << torch.arange(32, device="cuda")).sum(-1)
    bits = torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits).int()
    pos = s["len"][:, None] - s["count"][:, None] + sees.sum(-1).int() - 1
    s["mask"].copy_(torch.where(there[..., None], bits, s["mask"]))
    s["pos"].copy_(torch.where(there, pos, s["pos"]))
    return {"mask": s["mask"], "pos": s["pos"]}


def _plain_tree(s):
    case = s["case"]
    n, n_q, H, Hk, ps, D = case["n_seq"], case["n_q"], case["H"], case["Hk"], case["ps"], case["D"]
    G = H // Hk
    table, length = s["table"][:, 0].clamp(min=0).long(), s["len"].long()
    width = table.shape[1] * ps
    key = torch.arange(width, device="cuda")
    i = torch.arange(n_q, device="cuda")
    count = s["count"].long() if case["ragged"] else torch.full((n,), n_q, device="cuda")
    here = key < length
    k = s["k"][0][table].float().transpose(1, 2).reshape(n, Hk, width, D)
    q = s["q"][:, 0].float().view(n, n_q, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(n, Hk, n_q * G, D)
    z = torch.matmul(q, k.transpose(2, 3)).mul_(D ** -0.5).view(n, Hk, n_q, G, width)
    del k
    t = key - (length - count[:, None])  # which drafted token a key is
    if case["tree"]:
        word = torch.gather(s["mask"], 2, (t.clamp(0, n_q - 1) // 32)[:, None].expand(n, n_q, width))
        seen = (word >> (t.clamp(0, n_q - 1) % 32)[:, None].int() & 1) > 0
    else:
        seen = t[:, None] <= i[:, None]
    seen = ((t < 0)[:, None] | seen) & here[:, None]
    z.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    z = z.view(n, Hk, n_q * G, width)
    m = z.amax(-1, keepdim=True)
    m.masked_fill_(m == -math.inf, 0.0)
    p = z.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    v = s["v"][0][table].float().transpose(1, 2).reshape(n, Hk, width, D)
    v.masked_fill_(~here[:, None, :, None], 0.0)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.view(n, Hk, n_q, G, D).permute(0, 2, 1, 3, 4).reshape(n, n_q, H, D)
    lse = (m + total.log()).view(n, Hk, n_q, G).permute(0, 2, 1, 3).reshape(n, n_q, H)
    there = (i < count[:, None])[..., None]
    s["out"][:, 0] = torch.where(there[..., None], o.to(s["out"].dtype), s["out"][:, 0])
    s["lse"][:, 0] = torch.where(there, lse, s["lse"][:, 0])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_keep(s):
    case = s["case"]
    ps, table = case["ps"], s["table"][:, 0].long()
    ctx = s["len"].long() - case["n_q"]
    d = torch.arange(case["n_keep"], device="cuda")
    there = d < s["keep"][:, None]
    src, dst = ctx + s["path"].long(), (ctx + d).expand(-1, case["n_keep"])
    from_page, to_page = torch.gather(table, 1, src // ps)[there], torch.gather(table, 1, dst // ps)[there]
    from_row, to_row = (src % ps)[there], (dst % ps)[there]
    s["k"][:, to_page, :, to_row] = s["k"][:, from_page, :, from_row]
    s["v"][:, to_page, :, to_row] = s["v"][:, from_page, :, from_row]
    s["new_len"].copy_(ctx + s["keep"][:, None])
    return {"k": s["k"], "v": s["v"], "new_len": s["new_len"]}


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "rope":
        s["q_out"].copy_(_plain_rotate(s, s["q"], s["wq"], s["pos"]))
        s["k_out"].copy_(_plain_rotate(s, s["k"], s["wk"], s["pos"]))
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "append":
        return _plain_append(s)
    if kind == "masks":
        return _plain_masks(s)
    return _plain_tree(s) if kind == "tree" else _plain_keep(s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- from the definition, in 64 bits
def _exact_rotate(case, x, w, pos):
    """x [n][tokens][heads][D], pos [n][tokens]: each pair as a complex number, turned."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["D"] + EPS) * w.double()
    R = case["R"]
    angle = torch.from_numpy(pos[..., None].astype(np.float64) * _inv_freq(R)).cuda()[:, :, None]
    head = x[..., :R]
    pair = head.unflatten(-1, (R // 2, 2)) if case["interleaved"] else head.unflatten(-1, (2, R // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pair.contiguous()) * torch.polar(torch.full_like(angle, AMPLITUDE), angle)
    z = torch.view_as_real(z)
    z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., R:]], -1)


def _exact_append(case, seed):
    rows, k, v, count, length, table, (wq, wk) = _append_inputs(case, seed)
    n_new, H, Hk, ps = case["n_new"], case["H"], case["Hk"], case["ps"]
    pos = (length - count)[:, None] + np.arange(n_new)
    q, knew = _exact_rotate(case, rows[:, 0, :, :H], wq, pos), _exact_rotate(case, rows[:, 0, :, H:H + Hk], wk, pos)
    vnew = rows[:, 0, :, H + Hk:].double()
    k, v = k.double(), v.double()
    q_out = torch.zeros((case["n_seq"], 1, n_new, H, case["D"]), dtype=torch.float64, device="cuda")
    s, i = np.nonzero((np.arange(n_new) < count[:, None]) & (pos >= 0))
    token = pos[s, i]
    page, row = torch.from_numpy(table[s, token // ps]).cuda(), torch.from_numpy(token % ps).cuda()
    s, i = torch.from_numpy(s).cuda(), torch.from_numpy(i).cuda()
    q_out[s, 0, i] = q[s, i]
    k[0, page, :, row], v[0, page, :, row] = knew[s, i], vnew[s, i]
    return {"q": q_out, "k": k, "v": v}


def _exact_tree(case, seed):
    """Per sequence, its keys token by token."""
    q, k, v, count, ctx, table, sees = _tree_inputs(case, seed)
    H, Hk, ps = case["H"], case["Hk"], case["ps"]
    G, scale = H // Hk, 1.0 / math.sqrt(case["D"])
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:4], dtype=torch.float64, device="cuda")
    for r in range(case["n_seq"]):
        m, c = int(count[r]), int(ctx[r])
        token = np.arange(c + m)
        page, at = torch.from_numpy(table[r][token // ps]).cuda(), torch.from_numpy(token % ps).cuda()
        hidden = torch.zeros((m, c + m), dtype=torch.bool, device="cuda")
        hidden[:, c:] = torch.from_numpy(~sees[r if len(sees) > 1 else 0][:m, :m]).cuda()
        kk, vv = (x[0][page, :, at].double().transpose(0, 1) for x in (k, v))  # [heads][tokens][D]
        for g in range(G):
            heads = torch.arange(Hk, device="cuda") * G + g
            logit = scale * torch.einsum("ihd,hjd->hij", q[r, 0, :m][:, heads].double(), kk)
            logit[:, hidden] = -math.inf
            norm = torch.logsumexp(logit, 2)
            out[r, 0, :m, heads] = torch.einsum("hij,hjd->ihd", torch.exp(logit - norm[:, :, None]), vv)
            lse[r, 0, :m, heads] = norm.transpose(0, 1)
    return {"out": out, "lse": lse}


def exact(case, seed):
    """Rotations and attention; masks count and kept paths move: nothing is computed."""
    if case["kind"] == "rope":
        rows, pos, (wq, wk) = _rope_inputs(case, seed)
        H = case["H"]
        return {"q": _exact_rotate(case, rows[:, :, :H], wq, pos), "k": _exact_rotate(case, rows[:, :, H:], wk, pos)}
    if case["kind"] == "append":
        return _exact_append(case, seed)
    return _exact_tree(case, seed) if case["kind"] == "tree" else None


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Expected bytes (each input once, each output once) and flops of a pass."""
    kind, n = case["kind"], case["n_seq"]
    share = 0.5 if case.get("ragged") else 1.0
    if kind == "rope":
        rows = n * case["n_tok"] * (case["H"] + case["Hk"])
        return {"bytes": 4.0 * rows * case["D"] + 4.0 * n * case["n_tok"], "flops": 6.0 * rows * case["D"]}
    if kind == "append":
        rows = share * n * case["n_new"] * (case["H"] + 2 * case["Hk"])
        return {"bytes": 4.0 * rows * case["D"], "flops": 6.0 * rows * case["D"]}
    if kind == "masks":
        rows = share * n * case["n_tok"]
        return {"bytes": rows * (8.0 + 4.0 * -(-case["n_tok"] // 32)), "flops": 0}
    if kind == "tree":
        ctx, drafted = (case["ctx_lo"] + case["ctx_hi"]) / 2.0, max(1.0, share * case["n_q"])
        rows = n * drafted * case["H"]
        return {"bytes": n * (ctx + drafted) * case["Hk"] * 512.0 + rows * (4.0 * case["D"] + 4), "flops": 4.0 * case["D"] * rows * ctx}
    moved = n * max(0.5, case["n_keep"] / 2.0 - 0.5)
    return {"bytes": moved * case["layers"] * case["Hk"] * 1024.0, "flops": 0}
