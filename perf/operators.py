"""The paged K/V cache's operators, each in its plain form and as the package's calls.

Five kinds of passes over a cache whose pages the branches of a request share:

* ``attend``: attention of the sequences' newest tokens over their cached keys
  (``rps.rps_prefix_attention_fwd``); the pages that all sequences of a request
  share hold the same keys for each of them.
* ``branch``: the cache's part of a lookahead step: the valid branches fork from
  their request's base (``rps.rps_kv_fork_branches``), take pages for their
  tokens (``rps.rps_kv_resize``, which copies a shared last page before anyone
  writes into it), and the winner of the decision becomes the base
  (``rps.rps_kv_commit``).
* ``write``: new keys and values into the sequences' pages (``rps.rps_kv_write``).
* ``compact``: the live pages move to the lowest places (``rps.rps_kv_compact``).
* ``copy``: listed pages of one cache into another (``rps.rps_kv_copy_pages``).

``own`` selects the package's calls; otherwise ``run`` computes the same in
elementary torch operations, sums and softmax in 32 bits.

Where a pass changes the bookkeeping (reference counts, page tables, lengths),
it starts from the saved one, which is one small copy in both forms, so that
every pass does the same work. The pages that it writes are not among those
that it reads.
"""
import math

import numpy as np
import torch

own = False

D = 128
# No case costs more than the largest listed ones.
MAX_FLOPS = 290e9
MAX_CACHE_BYTES = 2.2e9
MAX_ROW_BYTES = 0.31e9


def _attend(name, n_req, n_branch, n_q, H, Hk, ps, shared, tail, causal, dtype):
    """shared, tail: ranges of a request's shared tokens and of a sequence's tokens after them."""
    c = dict(kind="attend", n_req=n_req, n_branch=n_branch, n_q=n_q, H=H, Hk=Hk, ps=ps, shared_lo=shared[0],
             shared_hi=shared[1], tail_lo=tail[0], tail_hi=tail[1], causal=causal, dtype=dtype)
    return dict(name=name, **c) if name else c


def _branch(name, n_req, n_branch, layers, Hk, ps, ctx, block, valid):
    """ctx: range of the context's tokens; valid: share of the branches that the step scores."""
    c = dict(kind="branch", n_req=n_req, n_branch=n_branch, layers=layers, Hk=Hk, ps=ps, ctx_lo=ctx[0], ctx_hi=ctx[1],
             block=block, valid=valid)
    return dict(name=name, **c) if name else c


def _write(name, n_seq, n_new, Hk, ps, length, dtype):
    c = dict(kind="write", n_seq=n_seq, n_new=n_new, Hk=Hk, ps=ps, len_lo=length[0], len_hi=length[1], dtype=dtype)
    return dict(name=name, **c) if name else c


def _compact(name, layers, n_pages, Hk, ps, live, n_seq):
    c = dict(kind="compact", layers=layers, n_pages=n_pages, Hk=Hk, ps=ps, live=live, n_seq=n_seq)
    return dict(name=name, **c) if name else c


def _copy(name, layers, n_pages, Hk, ps, count):
    c = dict(kind="copy", layers=layers, n_pages=n_pages, Hk=Hk, ps=ps, count=count)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one user's lookahead block: base and 8 branches of 32 tokens over a cached context, mostly latency
        _attend("attend-block", 1, 9, 32, 32, 32, 16, (328, 328), (32, 32), False, "bf16"),
        # token by token generation of many users behind one long system prompt, their own tails ragged
        _attend("attend-prompt", 1, 64, 1, 28, 4, 64, (8200, 8200), (5, 700), True, "bf16"),
        # lookahead blocks of a batch of requests, contexts ragged
        _attend("attend-serve", 64, 9, 32, 32, 32, 16, (200, 1200), (32, 32), False, "bf16"),
        # two requests' blocks over long contexts, heads that share keys, fp16
        _attend("attend-long", 2, 9, 32, 28, 4, 64, (24000, 32700), (32, 32), False, "f16"),
        # one lookahead step's forks and commit for one request
        _branch("branch-one", 1, 9, 4, 8, 16, (328, 328), 32, 1.0),
        # ... for a batch of requests, some branches not scored
        _branch("branch-serve", 64, 9, 4, 8, 16, (200, 900), 32, 0.75),
        # one token a sequence into its page
        _write("write-token", 16, 1, 4, 16, (1, 2000), "f16"),
        # the blocks of a batch's branches
        _write("write-serve", 576, 32, 32, 16, (40, 130), "bf16"),
        # a small cache, two fifths of it live
        _compact("compact-small", 4, 96, 4, 16, 0.4, 9),
        # a large one, half of it live, in odd sequences
        _compact("compact-large", 4, 8000, 8, 16, 0.5, 576),
        # a request's pages to another cache
        _copy("copy-request", 4, 256, 8, 16, 37),
        # a quarter of a large cache
        _copy("copy-large", 4, 4000, 8, 32, 1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "branch", "write", "compact", "copy"])
    while True:
        Hk = rng.choice([1, 2, 4, 8, 16, 28, 32])
        ps = rng.choice([16, 16, 32, 64, 128, 256])
        if kind == "attend":
            G = rng.choice([1, 1, 2, 4, 7, 8])
            n_q = rng.choice([1, 1, _log_int(rng, 2, 64), 32])
            hi = _log_int(rng, 16, 33000)
            lo = rng.choice([hi, max(1, hi // 6)])
            t_hi = n_q + rng.choice([0, 0, _log_int(rng, 1, 800)])
            t_lo = rng.choice([t_hi, n_q])
            c = _attend(None, _log_int(rng, 1, 64), _log_int(rng, 1, 64), n_q, G * Hk, Hk, ps, (lo, hi), (t_lo, t_hi),
                        rng.choice([True, False]), rng.choice(["bf16", "bf16", "f16"]))
            if Hk * G > 32 or work(c)["flops"] > MAX_FLOPS:
                continue
            pages = c["n_req"] * (hi // ps + 2 + c["n_branch"] * (t_hi // ps + 3))
            gathered = c["n_branch"] * (hi + t_hi + ps) * Hk * D * 4  # by the plain form, for keys and for values
            if pages * ps * Hk * D * 4 <= MAX_CACHE_BYTES / 2 and gathered <= 10e9:
                return c
        elif kind == "branch":
            hi = _log_int(rng, 40, 2000)
            c = _branch(None, _log_int(rng, 1, 64), rng.randint(2, 17), rng.choice([1, 2, 4]), Hk, ps,
                        (rng.choice([hi, max(1, hi // 5)]), hi), _log_int(rng, 1, 64), rng.choice([0.5, 0.75, 1.0]))
            if _branch_pages(c) * c["layers"] * ps * Hk * D * 4 <= MAX_CACHE_BYTES:
                return c
        elif kind == "write":
            n_new = rng.choice([1, _log_int(rng, 2, 64)])
            hi = n_new + _log_int(rng, 1, 1000)
            c = _write(None, _log_int(rng, 1, 600), n_new, Hk, ps, (n_new, hi), rng.choice(["bf16", "f16"]))
            if c["n_seq"] * n_new * Hk * D * 4 <= MAX_ROW_BYTES and c["n_seq"] * (hi // ps + 1) * ps * Hk * D * 4 <= MAX_CACHE_BYTES:
                return c
        else:
            layers, n_pages = rng.choice([1, 2, 4, 8]), _log_int(rng, 24, 30000)
            if layers * n_pages * ps * Hk * D * 4 > (1.0 if kind == "compact" else 0.5) * MAX_CACHE_BYTES:
                continue
            if kind == "compact":
                return _compact(None, layers, n_pages, Hk, ps, rng.choice([0.2, 0.5, 0.8]), _log_int(rng, 1, 600))
            return _copy(None, layers, n_pages, Hk, ps, rng.randint(1, max(1, n_pages // 4)))


# ---------------------------------------------------------------- inputs
def _dt(case):
    return torch.float16 if case.get("dtype") == "f16" else torch.bfloat16


def _normal(shape, dtype, g):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)


def _pages(tokens, ps):
    return -(-tokens // ps)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _book(n_pages, ps, table, length):
    """The bookkeeping as one tensor, and its views: reference counts, page tables, lengths."""
    ref = np.zeros(n_pages, np.int32)
    used = np.arange(table.shape[-1]) < np.maximum(_pages(length, ps), 0)[..., None]
    np.add.at(ref, table[used], 1)
    flat = _i32(np.concatenate([ref, table.ravel(), length.ravel()]))
    a, b = n_pages, n_pages + table.size
    return flat, flat[:a], flat[a:b].view(table.shape), flat[b:].view(length.shape)


def _attend_lengths(case, seed):
    """Shared tokens of each request, tokens of each sequence, page tables in a shuffled cache."""
    rs = np.random.default_rng(seed)
    n, nb, ps = case["n_req"], case["n_branch"], case["ps"]
    shared = rs.integers(case["shared_lo"], case["shared_hi"] + 1, n)
    length = shared[:, None] + rs.integers(case["tail_lo"], case["tail_hi"] + 1, (n, nb))
    width = int(_pages(case["shared_hi"] + case["tail_hi"], ps))
    table = np.full((n, nb, width), -1, np.int64)
    count = 0
    for r in range(n):
        both = int(shared[r]) // ps
        table[r, :, :both] = count + np.arange(both)
        count += both
        for b in range(nb):
            rest = int(_pages(int(length[r, b]), ps)) - both
            table[r, b, both:both + rest] = count + np.arange(rest)
            count += rest
    place = rs.permutation(count)
    return shared, length, np.where(table >= 0, place[table], -1), count


def _attend_inputs(case, seed):
    shared, length, table, count = _attend_lengths(case, seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = _normal((case["n_req"], case["n_branch"], case["n_q"], case["H"], D), _dt(case), g)
    q *= 2.0  # scores of about 2 nats' spread
    k = _normal((1, count, case["Hk"], case["ps"], D), _dt(case), g)
    v = _normal((1, count, case["Hk"], case["ps"], D), _dt(case), g)
    return q, k, v, shared, length, table


def _branch_pages(case):
    hi, ps = case["ctx_hi"] + case["block"], case["ps"]
    return case["n_req"] * (_pages(hi, ps) + case["n_branch"] * (_pages(case["block"], ps) + 2)) + 8


def _branch_book(case, seed):
    """Before the step: the bases hold their context and block, nothing else is live; and the step's inputs."""
    rs = np.random.default_rng(seed)
    n, nb, ps, block = case["n_req"], case["n_branch"], case["ps"], case["block"]
    n_pages = _branch_pages(case)
    ctx = rs.integers(case["ctx_lo"], case["ctx_hi"] + 1, n)
    width = int(_pages(case["ctx_hi"] + block, ps))
    table, length = np.full((n, nb, width), -1, np.int64), np.full((n, nb), -1, np.int64)
    place, count = rs.permutation(n_pages), 0
    for r in range(n):
        m = int(_pages(int(ctx[r]) + block, ps))
        table[r, 0, :m] = place[count:count + m]
        length[r, 0], count = ctx[r] + block, count + m
    valid = (rs.random((n, nb - 1)) < case["valid"]).astype(np.uint8)
    grown = np.where(np.concatenate([np.ones((n, 1)), valid], 1) > 0, (ctx + block)[:, None], -1)
    winner = np.full(n, -1, np.int64)
    for r in range(n):
        live = np.flatnonzero(valid[r])
        if len(live) and rs.random() < 0.8:
            winner[r] = rs.choice(live)
        elif rs.random() < 0.3:
            winner[r] = -2
    return n_pages, table, length, ctx, valid, grown, winner


def _compact_book(case, seed):
    """Sequences of odd lengths over a part of the cache; one in four shares half of its pages with the one before."""
    rs = np.random.default_rng(seed)
    n_pages, n_seq, ps = case["n_pages"], case["n_seq"], case["ps"]
    most = 2 * int(case["live"] * n_pages) // n_seq + 1  # pages of its own that a sequence may have
    sizes = rs.integers(0, most + 1, n_seq)
    sizes[0] = max(1, sizes[0])
    sizes = np.diff(np.minimum(np.concatenate([[0], np.cumsum(sizes)]), n_pages))
    place, at, rows = rs.permutation(n_pages), 0, []
    for s in range(n_seq):
        row = place[at:at + sizes[s]]
        at += sizes[s]
        if s and rs.random() < 0.25:
            row = np.concatenate([rows[-1][: len(rows[-1]) // 2], row])
        rows.append(row)
    table, length = np.full((n_seq, 1, 2 * most), -1, np.int64), np.full((n_seq, 1), -1, np.int64)
    for s, row in enumerate(rows):
        table[s, 0, : len(row)] = row
        length[s, 0] = max(0, len(row) * ps - int(rs.integers(0, ps))) if len(row) else rs.integers(-1, 1)
    return table, length


def _cache(case, n_pages, layers, g):
    shape = (layers, n_pages, case["Hk"], case["ps"], D)
    return _normal(shape, _dt(case), g), _normal(shape, _dt(case), g)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    rs = np.random.default_rng(seed + 2)
    kind, ps = case["kind"], case["ps"]
    s = {"case": case}
    if kind == "attend":
        s["q"], s["k"], s["v"], shared, length, table = _attend_inputs(case, seed)
        s["shared"] = _i32(shared)
        s["book"], s["ref"], s["table"], s["len"] = _book(s["k"].shape[1], ps, table, length)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(s["q"].shape[:4], dtype=torch.float32, device="cuda")
    elif kind == "branch":
        n_pages, table, length, ctx, valid, grown, winner = _branch_book(case, seed)
        s["book"], s["ref"], s["table"], s["len"] = _book(n_pages, ps, table, length)
        s["k"], s["v"] = _cache(case, n_pages, case["layers"], g)
        s["ctx"], s["grown"], s["winner"] = _i32(ctx), _i32(grown), _i32(winner)
        s["valid"] = torch.from_numpy(valid).cuda()
    elif kind == "write":
        n, n_new = case["n_seq"], case["n_new"]
        length = rs.integers(case["len_lo"], case["len_hi"] + 1, (n, 1))
        width = int(_pages(case["len_hi"], ps))
        n_pages = n * width
        table = np.full((n, 1, width), -1, np.int64)
        used = np.arange(width) < _pages(length, ps)[..., None]
        table[used] = rs.permutation(n_pages)[: used.sum()]
        s["book"], s["ref"], s["table"], s["len"] = _book(n_pages, ps, table, length)
        s["k"], s["v"] = _cache(case, n_pages, 1, g)
        s["k_new"] = _normal((n, 1, n_new, case["Hk"], D), _dt(case), g)
        s["v_new"] = _normal((n, 1, n_new, case["Hk"], D), _dt(case), g)
    elif kind == "compact":
        table, length = _compact_book(case, seed)
        s["book"], s["ref"], s["table"], s["len"] = _book(case["n_pages"], ps, table, length)
        s["k"], s["v"] = _cache(case, case["n_pages"], case["layers"], g)
        s["n_live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    else:
        s["k"], s["v"] = _cache(case, case["n_pages"], case["layers"], g)
        s["k2"], s["v2"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        s["src"] = _i32(rs.permutation(case["n_pages"])[: case["count"]])
        s["dst"] = _i32(rs.permutation(case["n_pages"])[: case["count"]])
    if "book" in s:
        s["book0"] = s["book"].clone()
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_2608_11742_gb300 import rps

    case = s["case"]
    if case["kind"] == "copy":
        s["from"], s["to"] = rps.KvCacheBuf.of_pages(s["k"], s["v"]), rps.KvCacheBuf.of_pages(s["k2"], s["v2"])
        return
    s["kv"] = rps.KvCacheBuf(s["k"], s["v"], s["ref"], s["table"], s["len"])
    if case["kind"] == "attend":
        n = rps.rps_prefix_attention_workspace_bytes(s["kv"], case["n_q"], case["H"])
    else:
        n = rps.rps_kv_workspace_bytes(s["kv"])
    s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------- the package's calls
def _run_own(s):
    from paper_2608_11742_gb300 import rps

    case, kind = s["case"], s["case"]["kind"]
    if kind == "attend":
        rps.rps_prefix_attention_fwd(s["q"], s["kv"], 0, s["out"], s["ws"], s["shared"], D ** -0.5, case["causal"], s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "write":
        rps.rps_kv_write(s["kv"], 0, s["k_new"], s["v_new"])
        return {"k": s["k"], "v": s["v"]}
    if kind == "copy":
        rps.rps_kv_copy_pages(s["from"], s["to"], s["src"], s["dst"])
        return {"k": s["k2"], "v": s["v2"]}
    s["book"].copy_(s["book0"])
    if kind == "branch":
        rps.rps_kv_fork_branches(s["kv"], s["valid"], s["ctx"], s["ws"])
        rps.rps_kv_resize(s["kv"], s["grown"], s["ws"])
        rps.rps_kv_commit(s["kv"], s["winner"], s["ws"])
        return {"book": s["book"], "k": s["k"], "v": s["v"]}
    rps.rps_kv_compact(s["kv"], s["n_live"], s["ws"])
    return {"book": s["book"], "n_live": s["n_live"], "k": s["k"], "v": s["v"]}


# ---------------------------------------------------------------- the plain forms
def _plain_attend(s):
    """Per request: the sequences' keys gathered to their places, masked softmax in fp32."""
    case = s["case"]
    nb, n_q, H, Hk, ps = case["n_branch"], case["n_q"], case["H"], case["Hk"], case["ps"]
    G, scale = H // Hk, D ** -0.5
    width = s["table"].shape[2] * ps
    key = torch.arange(width, device="cuda")
    for r in range(case["n_req"]):
        t = s["table"][r].clamp(min=0).long()
        n = s["len"][r].long()
        here = key < n[:, None]  # [nb][width]
        k = s["k"][0][t].float().transpose(1, 2).reshape(nb, Hk, width, D)
        v = s["v"][0][t].float().transpose(1, 2).reshape(nb, Hk, width, D)
        v.masked_fill_(~here[:, None, :, None], 0.0)
        q = s["q"][r].float().view(nb, n_q, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(nb, Hk, n_q * G, D)
        z = torch.matmul(q, k.transpose(2, 3)).mul_(scale).view(nb, Hk, n_q, G, width)
        limit = n[:, None].expand(nb, n_q)
        if case["causal"]:
            limit = limit - n_q + 1 + torch.arange(n_q, device="cuda")
        z.masked_fill_((key >= limit[:, :, None])[:, None, :, None, :], -math.inf)
        z = z.view(nb, Hk, n_q * G, width)
        m = z.amax(-1, keepdim=True)
        m.masked_fill_(m == -math.inf, 0.0)
        p = z.sub_(m).exp_()
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
        s["out"][r] = o.view(nb, Hk, n_q, G, D).permute(0, 2, 1, 3, 4).reshape(nb, n_q, H, D).to(s["out"].dtype)
        s["lse"][r] = (m + total.log()).view(nb, Hk, n_q, G).permute(0, 2, 1, 3).reshape(nb, n_q, H)
    return {"out": s["out"], "lse": s["lse"]}


def _held(s):
    """[sequences][width]: the places of the page table that hold a page."""
    ps = s["case"]["ps"]
    n = (s["len"].view(-1) + ps - 1).div(ps, rounding_mode="floor").clamp(min=0)
    return torch.arange(s["table"].shape[-1], device="cuda") < n[:, None]


def _plain_reorder(s, src, keep):
    """Every sequence takes the state of sequence src (-1: none), cut to keep tokens."""
    table, length = s["table"].view(-1, s["table"].shape[-1]), s["len"].view(-1)
    s["ref"].index_add_(0, table[_held(s)].long(), torch.full_like(table[_held(s)], -1))
    at = src.clamp(min=0).long()
    new_len = torch.where(src >= 0, length[at], -1)
    if keep is not None:
        new_len = torch.minimum(new_len, keep)
    rows = table[at]
    length.copy_(new_len)
    held = _held(s)
    table.copy_(torch.where(held, rows, -1))
    s["ref"].index_add_(0, table[held].long(), torch.ones_like(table[held]))


def _plain_resize(s, new_len):
    ps, ref = s["case"]["ps"], s["ref"]
    table, length = s["table"].view(-1, s["table"].shape[-1]), s["len"].view(-1)
    new_len = new_len.view(-1)
    # pages past the new end go back
    before = _held(s)
    grow = new_len > length
    old_len = length.clone()
    length.copy_(torch.minimum(length, new_len))
    gone = before & ~_held(s)
    ref.index_add_(0, table[gone].long(), torch.full_like(table[gone], -1))
    table.masked_fill_(gone, -1)
    # a shared last page that a sequence will write into is copied
    n_old = (old_len + ps - 1).div(ps, rounding_mode="floor").clamp(min=0)
    n_new = (new_len + ps - 1).div(ps, rounding_mode="floor").clamp(min=0)
    last = torch.gather(table, 1, (n_old - 1).clamp(min=0).long()[:, None])[:, 0]
    cow = grow & (old_len > 0) & (old_len % ps != 0) & (ref[last.clamp(min=0).long()] > 1)
    need = torch.where(grow, n_new - n_old, 0) + cow
    free = torch.nonzero(ref == 0)[:, 0].to(torch.int32)
    end = need.cumsum(0)
    fits = grow & (end <= free.numel())
    cow = cow & fits
    # entries that take a page: those from the first new one on, or from the copied one
    first = torch.where(cow, n_old - 1, n_old)
    col = torch.arange(table.shape[1], device="cuda")
    takes = fits[:, None] & (col >= first[:, None]) & (col < n_new[:, None])
    which = (end - need)[:, None] + col - first[:, None]
    table.copy_(torch.where(takes, free[which.clamp(0, max(0, free.numel() - 1)).long()] if free.numel() else table, table))
    ref.index_add_(0, table[takes].long(), torch.ones_like(table[takes]))
    ref.index_add_(0, last[cow].long(), torch.full_like(last[cow], -1))
    length.copy_(torch.where(fits, new_len, length))
    src, used = last[cow].long(), (old_len % ps)[cow]
    dst = torch.gather(table, 1, (n_old - 1).clamp(min=0).long()[:, None])[:, 0][cow].long()
    row = (torch.arange(ps, device="cuda") < used[:, None])[None, :, None, :, None]
    for x in (s["k"], s["v"]):
        x[:, dst] = torch.where(row, x[:, src], x[:, dst])


def _plain_compact(s):
    ref, table = s["ref"], s["table"].view(-1, s["table"].shape[-1])
    live = ref > 0
    n_live = int(live.sum())
    page = torch.arange(ref.numel(), device="cuda")
    src, dst = page[live & (page >= n_live)], page[~live & (page < n_live)]
    place = page.clone()
    place[src] = dst
    held = _held(s)
    table.copy_(torch.where(held, place[table.clamp(min=0).long()].to(torch.int32), table))
    ref[dst] = ref[src]
    ref[src] = 0
    for x in (s["k"], s["v"]):
        x[:, dst] = x[:, src]
    s["n_live"].fill_(n_live)


def _plain_write(s):
    ps, n_new = s["case"]["ps"], s["case"]["n_new"]
    table, length = s["table"].view(-1, s["table"].shape[-1]), s["len"].view(-1).long()
    pos = length[:, None] - n_new + torch.arange(n_new, device="cuda")
    page = torch.gather(table.long(), 1, pos.clamp(min=0).div(ps, rounding_mode="floor"))
    for x, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
        x[0][page, :, pos % ps] = new[:, 0]


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "attend":
        return _plain_attend(s)
    if kind == "write":
        _plain_write(s)
        return {"k": s["k"], "v": s["v"]}
    if kind == "copy":
        src, dst = s["src"].long(), s["dst"].long()
        s["k2"][:, dst] = s["k"][:, src]
        s["v2"][:, dst] = s["v"][:, src]
        return {"k": s["k2"], "v": s["v2"]}
    s["book"].copy_(s["book0"])
    if kind == "branch":
        n, nb = s["len"].shape
        base = torch.arange(n, dtype=torch.int32, device="cuda")[:, None] * nb
        far = torch.full((n, 1), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
        src = torch.cat([base, torch.where(s["valid"] > 0, base, -1)], 1)
        keep = torch.cat([far, s["ctx"][:, None].expand(n, nb - 1)], 1)
        _plain_reorder(s, src.view(-1), keep.reshape(-1))
        _plain_resize(s, s["grown"])
        src = torch.full((n, nb), -1, dtype=torch.int32, device="cuda")
        src[:, :1] = base + torch.where(s["winner"] >= 0, s["winner"] + 1, 0)[:, None]
        _plain_reorder(s, src.view(-1), None)
        return {"book": s["book"], "k": s["k"], "v": s["v"]}
    _plain_compact(s)
    return {"book": s["book"], "n_live": s["n_live"], "k": s["k"], "v": s["v"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- from the definition, in 64 bits
def exact(case, seed):
    """Attention: per sequence, its keys token by token in fp64. The others move and count: nothing is computed."""
    if case["kind"] != "attend":
        return None
    q, k, v, _, length, table = _attend_inputs(case, seed)
    n_q, H, Hk, ps = case["n_q"], case["H"], case["Hk"], case["ps"]
    G, scale = H // Hk, 1.0 / math.sqrt(D)
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:4], -math.inf, dtype=torch.float64, device="cuda")
    per = max(1, int(1e8) // (n_q * G * int(length.max())))  # heads at a time
    for r in range(case["n_req"]):
        for b in range(case["n_branch"]):
            n = int(length[r, b])
            token = np.arange(n)
            page = torch.from_numpy(table[r, b][token // ps]).cuda()
            at = torch.from_numpy(token % ps).cuda()
            mask = None
            if case["causal"]:
                last = torch.arange(n - n_q, n, device="cuda")
                mask = torch.arange(n, device="cuda")[None, :] > last[:, None]
            for h0 in range(0, Hk, per):
                h1 = min(Hk, h0 + per)
                kk = k[0, page, h0:h1, at].double().transpose(0, 1)  # [heads][n][D]
                vv = v[0, page, h0:h1, at].double().transpose(0, 1)
                for g in range(G):
                    heads = torch.arange(h0, h1, device="cuda") * G + g
                    qq = q[r, b][:, heads].double().transpose(0, 1)  # [heads][n_q][D]
                    logit = scale * torch.einsum("hid,hjd->hij", qq, kk)
                    if mask is not None:
                        logit[:, mask] = -math.inf
                    norm = torch.logsumexp(logit, 2)
                    weight = torch.exp(logit - norm[:, :, None])
                    out[r, b, :, heads] = torch.einsum("hij,hjd->hid", weight, vv).transpose(0, 1)
                    lse[r, b, :, heads] = norm.transpose(0, 1)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Expected bytes (each input once, each output once) and flops of a pass."""
    kind, ps = case["kind"], case["ps"]
    row = 2 * 2 * D  # one token of one head, keys and values
    if kind == "attend":
        shared, tail = (case["shared_lo"] + case["shared_hi"]) / 2.0, (case["tail_lo"] + case["tail_hi"]) / 2.0
        n_seq = case["n_req"] * case["n_branch"]
        cached = case["n_req"] * (shared + case["n_branch"] * tail) * case["Hk"]
        tokens = n_seq * case["n_q"] * case["H"]
        seen = shared + tail - ((case["n_q"] - 1) / 2.0 if case["causal"] else 0.0)
        return {"bytes": cached * row + tokens * (4.0 * D + 4), "flops": 4.0 * D * tokens * seen}
    if kind == "branch":
        # the valid branches' shared last pages (half a page each, all but one time in ps), and the tables
        n = case["n_req"] * (case["n_branch"] - 1) * case["valid"]
        distinct = case["n_req"] * (case["ps"] - 1) / 2.0
        data = (n * (ps - 1) / 2.0 + distinct) * case["layers"] * case["Hk"] * row
        width = _pages((case["ctx_lo"] + case["ctx_hi"]) / 2.0 + case["block"], ps)
        return {"bytes": data + 4.0 * (2 * case["n_req"] * case["n_branch"] * width + 2 * _branch_pages(case)), "flops": 0}
    if kind == "write":
        return {"bytes": 2.0 * case["n_seq"] * case["n_new"] * case["Hk"] * row, "flops": 0}
    page = case["layers"] * ps * case["Hk"] * row
    if kind == "compact":
        moved = case["live"] * (1.0 - case["live"]) * case["n_pages"]
        return {"bytes": 2.0 * moved * page + 4.0 * (2 * case["n_pages"] + 2 * case["live"] * case["n_pages"]), "flops": 0}
    return {"bytes": 2.0 * case["count"] * page + 8.0 * case["count"], "flops": 0}
