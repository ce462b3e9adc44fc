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
// Work. Row tiles are numbered through (request, head, row tile) and have costs: so much
// for the row tile and so much for each of its key tiles. The n CTAs take equal parts
// (to one tile) of the sum of the costs, so a row tile may be spread over several
// CTAs, whose partial results are joined afterwards.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define PREFIX_HD __host__ __device__ __forceinline__
#else
#define PREFIX_HD inline
#endif

namespace rps {
namespace prefix {

constexpr int kRows = 128;     // rows of a row tile, keys of a key tile
constexpr int kMaxCtas = 160;  // CTAs of a call, and cut row tiles that are listed

// Division of 0 <= n < 2^31 by a constant d: with l = ceil(log2 d) and mul = ceil(2^(31 + l) / d),
// n mul / 2^(31 + l) exceeds n / d by less than n / 2^31 / d * (d / 2^l) < 1 / d, so its floor is
// the quotient. (The compiler's code for a division by a variable is several times as long; the
// roles' code has to fit the instruction cache together.)
struct Div {
    uint32_t mul, shift;
};
PREFIX_HD Div make_div(int d) {
    Div v;
    uint32_t l = 0;
    while ((int64_t{1} << l) < d) ++l;
    v.shift = 31 + l;
    v.mul = static_cast<uint32_t>(((uint64_t{1} << v.shift) + static_cast<uint64_t>(d) - 1) / static_cast<uint64_t>(d));
    return v;
}
PREFIX_HD int quotient(int n, const Div &v) {
    return static_cast<int>(static_cast<uint64_t>(static_cast<uint32_t>(n)) * v.mul >> v.shift);
}

struct Shape {
    int32_t n_req, n_branch, n_q, n_tokens;   // n_tokens = n_branch * n_q
    int32_t heads, group;                     // cache heads, query heads per cache head
    int32_t tokens, row_tiles;                // tokens of a row tile, row tiles of a (request, head)
    int32_t page, slot, sub, spt;             // tokens of a page, of a slot; slots per page, per key tile
    int32_t page_log, slot_log, sub_log, spt_log;  // all four are powers of two
    int32_t n_pages, max_pages;
    int32_t causal;
    Div by_n_q, by_group, by_row_tiles;
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
    s.page_log = s.slot_log = s.sub_log = s.spt_log = 0;
    while ((1 << s.page_log) < s.page) ++s.page_log;
    while ((1 << s.slot_log) < s.slot) ++s.slot_log;
    while ((1 << s.sub_log) < s.sub) ++s.sub_log;
    while ((1 << s.spt_log) < s.spt) ++s.spt_log;
    s.by_n_q = make_div(n_q);
    s.by_group = make_div(group);
    s.by_row_tiles = make_div(s.row_tiles);
    s.n_pages = n_pages;
    s.max_pages = max_pages;
    s.causal = causal;
    return s;
}

PREFIX_HD int slots_of(const Shape &s, int len) { return (len + s.slot - 1) >> s.slot_log; }
PREFIX_HD int tiles_of(const Shape &s, int slots) { return (slots + s.spt - 1) >> s.spt_log; }

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
    r.b0 = quotient(r.tok0, s.by_n_q);
    r.nb = quotient(r.tok0 + r.n_tok - 1, s.by_n_q) - r.b0 + 1;
    return r;
}

// Sums over the sequences of a row tile from which its key tiles follow.
struct KeySum {
    int32_t present, slots, min_pages;  // sequences there; their slots; whole pages of the shortest
};
PREFIX_HD void add_sequence(const Shape &s, KeySum &k, int len) {
    k.present += len >= 0;  // (an absent one's -1 makes no slot: slots are 16 tokens at least)
    k.slots += slots_of(s, len);
    k.min_pages = imin(k.min_pages, len >= 0 ? len >> s.page_log : INT32_MAX);
}
// Slots that are read once for the row tile's sequences: whole pages inside the shared length and inside each of them.
PREFIX_HD int shared_slots(const Shape &s, const KeySum &k, int shared_len) {
    return k.present ? imin(imax(0, shared_len) >> s.page_log, k.min_pages) << s.sub_log : 0;
}
// Key tiles: none where no sequence is there, at least one else (rows that see nothing are written too).
struct Tiles {
    int32_t shared, own;
};
PREFIX_HD Tiles key_tiles(const Shape &s, const KeySum &k, int shared) {
    Tiles t;
    t.shared = t.own = 0;
    if (!k.present) return t;
    t.shared = tiles_of(s, shared);
    t.own = tiles_of(s, k.slots - k.present * shared);
    if (t.shared + t.own == 0) t.own = 1;
    return t;
}

// Costs, in quarters of a shared tile's 1700 cycles: an own tile takes 2500 (its product writes the
// rows of one sequence at a time); the change from a row tile to the next 2800 (the product waits for
// the read-out), and a cut one's parts are written and joined. With row tiles at 6 instead of 10, 64
// sequences of one prompt took 30.2 us instead of 28.8, 64 requests of 9 branches 396 instead of 399.
constexpr int kSharedCost = 4, kOwnCost = 6, kRowCost = 10;
PREFIX_HD int cost_of(Tiles t) {
    return t.shared + t.own ? kRowCost + kSharedCost * t.shared + kOwnCost * t.own : 0;
}
// Where a row tile's tiles lie in its costs: tile k belongs to the range (y0, y1] that holds place(t, k),
// the middle of its cost (of the first one's and the row tile's). No two neighbours, of the next row tile
// too, are more than kWidest apart.
constexpr int kFirstPlace = (kRowCost + kSharedCost) / 2, kWidest = kRowCost + kOwnCost;
PREFIX_HD int place(Tiles t, int k) {
    if (k == 0) return kFirstPlace;
    return kRowCost + (k < t.shared ? kSharedCost * k + kSharedCost / 2
                                    : kSharedCost * t.shared + kOwnCost * (k - t.shared) + kOwnCost / 2);
}
// The tiles whose places are at most y.
PREFIX_HD int reach(Tiles t, int64_t y) {
    if (y < kFirstPlace || t.shared + t.own == 0) return 0;
    if (y >= cost_of(t)) return t.shared + t.own;
    const int x = static_cast<int>(y) - kRowCost, own = x - kSharedCost * t.shared;
    const int k = own < 0 ? (x + kSharedCost / 2) / kSharedCost : t.shared + (own + kOwnCost / 2) / kOwnCost;
    return imax(1, imin(k, t.shared + t.own));
}

// The n CTAs' ranges of the costs: `base` each, the first `extra` one more. (By 16-bit digits:
// n is small.) A CTA whose range is at least kWidest long has a tile.
struct Ranges {
    int64_t base;
    int32_t extra, n;
};
PREFIX_HD Ranges make_ranges(int64_t work, int n) {
    Ranges r;
    const uint32_t d = static_cast<uint32_t>(n);  // at most 2^16
    uint64_t q = 0;
    uint32_t rem = 0;
#pragma unroll 1
    for (int at = 48; at >= 0; at -= 16) {
        const uint32_t part = (rem << 16) | static_cast<uint32_t>(static_cast<uint64_t>(work) >> at & 0xffffu);
        q = q << 16 | part / d;
        rem = part % d;
    }
    r.base = static_cast<int64_t>(q);
    r.extra = static_cast<int32_t>(rem);
    r.n = n;
    return r;
}
PREFIX_HD int64_t range_start(const Ranges &r, int c) { return c * r.base + imin(c, r.extra); }
// The CTA in whose range [start, ..) x lies.
PREFIX_HD int cta_of(const Ranges &r, int64_t x) {
    int lo = 0, hi = r.n;
#pragma unroll 1
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (range_start(r, mid) <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// The list of cut row tiles, and the blocks that join their parts, one an entry. Entries are by
// row tile while there are at most kMaxCtas of them (more than the CTAs of a card with fewer SMs:
// each row tile has a block, not each CTA), else by the CTA that takes the first part: one CTA
// begins at most one cut row tile, its last.
struct CutList {
    int32_t by_tile, blocks;
};
PREFIX_HD CutList cut_list(int64_t row_tiles, int ctas) {
    CutList l;
    l.by_tile = row_tiles <= kMaxCtas;
    l.blocks = l.by_tile ? static_cast<int32_t>(row_tiles) : ctas;
    return l;
}

// The sequence i of [0, nb) that holds own slot x (off[i] <= x < off[i + 1]; x < off[nb]).
PREFIX_HD int slot_owner(const int32_t *off, int nb, int x) {
    int lo = 0, hi = nb;
#pragma unroll 1
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
    const int first = (j - shared_tiles) * s.spt, x = first + (kk * 16 >> s.slot_log);
    if (x >= off[r.nb]) return st;
    const int i = slot_owner(off, r.nb, x), inner = kk * 16 & (s.slot - 1);
    const int key = (x - off[i] + shared) * s.slot + inner;
    st.who = i;
    st.keys = imax(0, imin(16, len[i] - key));
    const int t0 = imax(0, (r.b0 + i) * s.n_q - r.tok0), t1 = imin(r.n_tok, (r.b0 + i + 1) * s.n_q - r.tok0);
    st.r0 = t0 * s.group;
    st.r1 = t1 * s.group;
    const int begin = imax(off[i], first);  // the sequence's first slot in this tile
    const int prev = j - 2, from = shared_tiles + (off[i] >> s.spt_log), oldest = j0 + ((j - j0) & 1);
    const bool touched = prev >= j0 && (prev >= from || oldest < shared_tiles);
    st.fresh = x == begin && inner == 0 && !touched;
    return st;
}

}  // namespace prefix
}  // namespace rps
