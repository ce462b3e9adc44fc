// prefix_split.h -- how the attention over the paged cache cuts its work, in plain
// C++ (host and device), so that the cut can be checked on the host.
//
// Rows. The query rows of one (request, cache head) are its n_branch * n_q tokens
// times the `group` query heads that share the head; a row tile takes as many
// whole tokens as fit 128 rows (row = token in the tile * group + head in group).
// Keys. The cache is read in slots: `slot` = min(page_size, 128) keys of one page;
// a key tile is 128 / slot slots. The key tiles of a row tile are those of the
// shared slots (the leading pages that all its sequences hold), then those of its
// sequences' own slots, one sequence after another with no gap (a sequence's last
// slot may be partly filled).
// Work. Key tiles are numbered through (request, head, row tile, key tile), and
// CTA c of n <= W takes tiles [c W / n, (c + 1) W / n): equal parts, so a row tile may
// be spread over several CTAs, whose partial results are joined afterwards.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define PREFIX_HD __host__ __device__ __forceinline__
#else
#define PREFIX_HD inline
#endif

namespace rps {
namespace prefix {

constexpr int kRows = 128;  // rows of a row tile, keys of a key tile

struct Shape {
    int32_t n_req, n_branch, n_q, n_tokens;   // n_tokens = n_branch * n_q
    int32_t heads, group;                     // cache heads, query heads per cache head
    int32_t tokens, row_tiles;                // tokens of a row tile, row tiles of a (request, head)
    int32_t page, slot, sub, spt;             // tokens of a page, of a slot; slots per page, per key tile
    int32_t n_pages, max_pages;
    int32_t causal;
};

PREFIX_HD int imin(int a, int b) { return a < b ? a : b; }
PREFIX_HD int imax(int a, int b) { return a > b ? a : b; }
PREFIX_HD int ceil_div(int a, int b) { return (a + b - 1) / b; }

PREFIX_HD Shape make_shape(int n_req, int n_branch, int n_q, int heads, int group, int page, int n_pages,
                           int max_pages, int causal) {
    Shape s;
    s.n_req = n_req;
    s.n_branch = n_branch;
    s.n_q = n_q;
    s.n_tokens = n_branch * n_q;
    s.heads = heads;
    s.group = group;
    s.tokens = imin(kRows / group, s.n_tokens);
    s.row_tiles = ceil_div(s.n_tokens, s.tokens);
    s.page = page;
    s.slot = imin(page, kRows);
    s.sub = page / s.slot;
    s.spt = kRows / s.slot;
    s.n_pages = n_pages;
    s.max_pages = max_pages;
    s.causal = causal;
    return s;
}

// A sequence's length as it is used: -1 absent, at most what its table row holds.
PREFIX_HD int used_len(const Shape &s, int len) { return len < 0 ? -1 : imin(len, s.max_pages * s.page); }

// Row tile rt: tokens [tok0, tok0 + n_tok) of the request, sequences [b0, b0 + nb).
struct RowTile {
    int32_t tok0, n_tok, b0, nb;
};
PREFIX_HD RowTile row_tile(const Shape &s, int rt) {
    RowTile r;
    r.tok0 = rt * s.tokens;
    r.n_tok = imin(s.tokens, s.n_tokens - r.tok0);
    r.b0 = r.tok0 / s.n_q;
    r.nb = (r.tok0 + r.n_tok - 1) / s.n_q - r.b0 + 1;
    return r;
}

// Sums over the sequences of a row tile from which its key tiles follow.
struct KeySum {
    int32_t present, slots, min_pages;  // sequences there; their slots; whole pages of the shortest
};
PREFIX_HD void add_sequence(const Shape &s, KeySum &k, int len) {
    if (len < 0) return;
    ++k.present;
    k.slots += ceil_div(len, s.slot);
    k.min_pages = imin(k.min_pages, len / s.page);
}
// Slots that are read once for all: whole pages inside the shared length and inside every sequence.
PREFIX_HD int shared_slots(const Shape &s, const KeySum &k, int shared_len) {
    return k.present ? imin(imax(0, shared_len) / s.page, k.min_pages) * s.sub : 0;
}
// Key tiles: none where no sequence is there, at least one else (rows that see nothing are written too).
PREFIX_HD int key_tiles(const Shape &s, const KeySum &k, int shared) {
    if (!k.present) return 0;
    const int own = k.slots - k.present * shared;
    return imax(1, ceil_div(shared, s.spt) + ceil_div(own, s.spt));
}

PREFIX_HD int64_t range_start(int c, int64_t work, int n) { return static_cast<int64_t>(c) * work / n; }
// The CTA that takes tile x - 1 (x >= 1).
PREFIX_HD int last_cta(int64_t x, int64_t work, int n) { return static_cast<int>((x * n - 1) / work); }

// The sequence i of [0, nb) that holds own slot x (off[i] <= x < off[i + 1]; x < off[nb]).
PREFIX_HD int slot_owner(const int32_t *off, int nb, int x) {
    int lo = 0, hi = nb;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// Keys [0, row_limit) of a sequence of len tokens that query i of it sees.
PREFIX_HD int row_limit(const Shape &s, int len, int i) {
    return len < 0 ? 0 : s.causal ? imax(0, len - s.n_q + i + 1) : len;
}

// Columns [lo, hi) of key tile j that a row sees: its sequence's own slots begin at `off`, `limit` is its row_limit.
struct Columns {
    int32_t lo, hi;
};
PREFIX_HD Columns row_columns(const Shape &s, int j, int shared_tiles, int shared, int off, int limit) {
    Columns c;
    if (j < shared_tiles) {
        c.lo = 0;
        c.hi = imin(kRows, imin(shared * s.slot, limit) - j * kRows);
    } else {
        const int first = (off - (j - shared_tiles) * s.spt) * s.slot;  // the column of the sequence's first own key
        c.lo = imax(0, first);
        c.hi = imin(kRows, first + limit - shared * s.slot);
    }
    return c;
}

// The 16 keys of step kk of own key tile j (the product's K extent): those of
// sequence `who`, `keys` of them filled (0: the step is left out); rows [r0, r1)
// of the tile are that sequence's. `fresh`: nothing was added to these rows yet by
// tiles of the same parity of the piece [j0, ..): the step overwrites.
struct Step {
    int32_t who, keys, r0, r1, fresh;
};
PREFIX_HD Step own_step(const Shape &s, const RowTile &r, const int32_t *off, const int32_t *len, int shared_tiles,
                        int shared, int j0, int j, int kk) {
    Step st;
    st.who = st.keys = st.r0 = st.r1 = st.fresh = 0;
    const int first = (j - shared_tiles) * s.spt, x = first + kk * 16 / s.slot;
    if (x >= off[r.nb]) return st;
    const int i = slot_owner(off, r.nb, x), inner = kk * 16 % s.slot;
    const int key = (x - off[i] + shared) * s.slot + inner;
    st.who = i;
    st.keys = imax(0, imin(16, len[i] - key));
    const int t0 = imax(0, (r.b0 + i) * s.n_q - r.tok0), t1 = imin(r.n_tok, (r.b0 + i + 1) * s.n_q - r.tok0);
    st.r0 = t0 * s.group;
    st.r1 = t1 * s.group;
    const int begin = imax(off[i], first);  // the sequence's first slot in this tile
    const int prev = j - 2, from = shared_tiles + off[i] / s.spt, oldest = j0 + ((j - j0) & 1);
    const bool touched = prev >= j0 && (prev >= from || oldest < shared_tiles);
    st.fresh = x == begin && inner == 0 && !touched;
    return st;
}

}  // namespace prefix
}  // namespace rps
