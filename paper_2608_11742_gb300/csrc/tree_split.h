// tree_split.h -- how the attention of drafted tokens cuts its work, in plain C++ (host
// and device), so that the cut can be checked on the host.
//
// Rows. The query rows of one (sequence, cache head) are its drafted tokens times the
// `group` query heads that share the head; a row tile takes as many whole tokens as fit
// 128 rows (row = token in the tile * group + head in group). A unit is a pair of
// neighbouring row tiles, or a last one alone: a pair reads the keys once.
// Keys. A key tile is 128 tokens of the sequence. A unit takes the key tiles up to the
// last key that one of its rows sees; at least one (rows that see nothing are written too).
// Work. Units are numbered through (sequence, head, pair) and have places: kTileCost or
// kPairCost for each of their key tiles, and kUnitCost or kPairUnitCost behind them. The n CTAs take equal parts
// of all places, a key tile goes where its first place is; so a unit may be spread over
// several CTAs, whose partial results are joined afterwards.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "prefix_split.h"

namespace rps {
namespace tree {

using prefix::ceil_div;
using prefix::Div;
using prefix::imax;
using prefix::imin;
using prefix::quotient;

constexpr int kRows = 128;     // rows of a row tile, keys of a key tile
constexpr int kMaxCtas = 160;  // CTAs of a call
// Costs, in thirds of a key tile of one row tile: fitted to the times of 152 CTAs, which take 1.07 us for
// such a tile, 1.65 for one of a pair, 2.0 to 2.5 for a unit's begin and end, 4.1 for a pair's. (By
// numbers of key tiles, 64 sequences of 1 to 32 drafted tokens, 32/4 heads: the first CTA ended after
// 45 us, the last after 80.)
constexpr int kTileCost = 3, kPairCost = 5, kUnitCost = 6, kPairUnitCost = 11;
// Cutting a unit costs what its parts take to be written and joined, as much as three key tiles: where
// every unit has a CTA of its own and none costs by more than that more than the equal shares, none is cut.
constexpr int kCutCost = 3 * kTileCost;

struct Shape {
    int32_t n_seq, n_q, heads, group;  // heads of the cache, query heads of each
    int32_t tokens;                    // of a row tile
    int32_t pairs;                     // units of a (sequence, head) at most
    int32_t page_log, max_pages, n_pages;
    int32_t chain;                     // no mask: token i sees drafted tokens 0..i
    Div by_group, by_tokens;
};

PREFIX_HD Shape make_shape(int n_seq, int n_q, int heads, int group, int page, int n_pages, int max_pages, int chain) {
    Shape s;
    s.n_seq = n_seq;
    s.n_q = n_q;
    s.heads = heads;
    s.group = group;
    s.tokens = imin(kRows / group, n_q);
    s.pairs = ceil_div(ceil_div(n_q, s.tokens), 2);
    s.page_log = 0;
    while ((1 << s.page_log) < page) ++s.page_log;
    s.max_pages = max_pages;
    s.n_pages = n_pages;
    s.chain = chain;
    s.by_group = prefix::make_div(group);
    s.by_tokens = prefix::make_div(s.tokens);
    return s;
}

// A sequence as it is used: its tokens (-1 absent, at most what its table row holds), and how
// many of the last ones are queries.
struct Seq {
    int32_t len, count;
};
PREFIX_HD Seq used_seq(const Shape &s, int len, int count) {
    Seq q;
    q.len = len < 0 ? -1 : imin(len, s.max_pages << s.page_log);
    q.count = len < 0 ? 0 : imax(0, imin(count, s.n_q));
    return q;
}

// Units of a head of the sequence.
PREFIX_HD int pairs_of(const Shape &s, const Seq &q) {
    return (quotient(q.count + s.tokens - 1, s.by_tokens) + 1) >> 1;
}
// Row tiles of unit p (1 or 2), and its key tiles.
PREFIX_HD int row_tiles_of(const Shape &s, const Seq &q, int p) { return q.count > (2 * p + 1) * s.tokens ? 2 : 1; }
PREFIX_HD int tiles_of(const Shape &s, const Seq &q, int p) {
    const int last = s.chain ? imin(q.count, (2 * p + 2) * s.tokens) : q.count;  // queries before it see no further
    return imax(1, (q.len - q.count + last + kRows - 1) >> 7);
}

PREFIX_HD int tile_cost(int row_tiles) { return row_tiles > 1 ? kPairCost : kTileCost; }
PREFIX_HD int unit_cost(int row_tiles) { return row_tiles > 1 ? kPairUnitCost : kUnitCost; }
PREFIX_HD int cost_of(const Shape &s, const Seq &q, int p) {
    const int rt = row_tiles_of(s, q, p);
    return tiles_of(s, q, p) * tile_cost(rt) + unit_cost(rt);
}

// The bits of keys [key, key + 32) that query i of the sequence sees, for a chain.
PREFIX_HD uint32_t low_ones(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1; }
PREFIX_HD uint32_t chain_bits(const Seq &q, int i, int key) {
    return low_ones(imin(q.len, q.len - q.count + i + 1) - key);
}
// The same from a mask of drafted tokens: word(w) gives word w of the query's row, for
// 0 <= w < ceil(n_q / 32).
template <typename Word>
PREFIX_HD uint32_t mask_bits(const Seq &q, int key, Word word) {
    const int b = key - (q.len - q.count);  // the drafted token that the first key is
    if (b <= -32) return ~0u;
    const auto at = [&](int w) -> uint32_t {
        if (w < 0) return ~0u;
        if (w * 32 >= q.count) return 0u;
        return word(w) & low_ones(q.count - w * 32);
    };
    const int w = b >> 5, shift = b & 31;
    const uint32_t lo = at(w);
    return shift ? lo >> shift | at(w + 1) << (32 - shift) : lo;
}

// The n CTAs' ranges of the places: `base` each, the first `extra` one more. With kPairCost places and
// more in each, one that lies inside a unit's key tiles has a tile.
struct Ranges {
    int64_t base;
    int32_t extra, n;
};
// (A division of 32 bits where they are enough: one of 64 takes several times as long.)
PREFIX_HD int64_t divide(int64_t x, int64_t d) {
    return (x | d) >> 32 ? x / d : static_cast<int64_t>(static_cast<uint32_t>(x) / static_cast<uint32_t>(d));
}
PREFIX_HD Ranges make_ranges(int64_t work, int n) {
    Ranges r;
    r.base = divide(work, n);
    r.extra = static_cast<int32_t>(work - r.base * n);
    r.n = n;
    return r;
}
PREFIX_HD int64_t range_start(const Ranges &r, int c) { return c * r.base + imin(c, r.extra); }
// The CTA in whose range place x lies (base > 0).
PREFIX_HD int cta_of(const Ranges &r, int64_t x) {
    const int64_t wide = r.extra * (r.base + 1);
    return static_cast<int>(x < wide ? divide(x, r.base + 1) : r.extra + divide(x - wide, r.base));
}

// A walk through the units of a CTA's range, piece by piece.
struct Walk {
    int32_t s, h, p, j;  // the next unit, and how many of its places are taken
    int64_t left;        // places of the range
};
struct Piece {
    int32_t s, h, p, rt;        // rt: row tiles
    int32_t j0, j1, tiles;      // its key tiles, of the unit's
    int32_t part;               // -1: the whole unit; 1: its first tiles; 0: later ones
    int32_t to_last;            // places from the range's end to the unit's last tile, of its first tiles
    Seq q;
};
// The next piece (false: there is none). seq(s) gives a sequence as used.
template <typename SeqOf>
PREFIX_HD bool next_piece(const Shape &s, Walk &w, Piece &x, SeqOf seq) {
#pragma unroll 1
    while (w.left > 0 && w.s < s.n_seq) {
        x.q = seq(w.s);
        const int pairs = pairs_of(s, x.q);
        if (pairs == 0) {
            ++w.s;
            continue;
        }
        x.s = w.s;
        x.h = w.h;
        x.p = w.p;
        x.rt = row_tiles_of(s, x.q, w.p);
        x.tiles = tiles_of(s, x.q, w.p);
        const int each = tile_cost(x.rt), cost = x.tiles * each + unit_cost(x.rt), rest = cost - w.j;
        const int take = w.left < rest ? static_cast<int>(w.left) : rest, end = w.j + take;
        x.j0 = imin(x.tiles, ceil_div(w.j, each));
        x.j1 = imin(x.tiles, ceil_div(end, each));
        x.part = x.j0 > 0 ? 0 : x.j1 < x.tiles ? 1 : -1;
        x.to_last = (x.tiles - 1) * each - end;
        w.left -= take;
        w.j += take;
        if (w.j == cost) {
            w.j = 0;
            if (++w.p == pairs) {
                w.p = 0;
                if (++w.h == s.heads) {
                    w.h = 0;
                    ++w.s;
                }
            }
        }
        if (x.j1 > x.j0) return true;
    }
    return false;
}
// The walk that begins `rem` places into sequence `at`, `left` places long. (rem is inside the sequence.)
PREFIX_HD Walk begin_walk(const Shape &s, int at, const Seq &q, int64_t rem, int64_t left) {
    Walk w;
    const int pairs = pairs_of(s, q);
    int64_t head = 0;
#pragma unroll 1
    for (int p = 0; p < pairs; ++p) head += cost_of(s, q, p);
    w.s = at;
    w.h = static_cast<int>(divide(rem, head));
    rem -= w.h * head;
    w.p = 0;
#pragma unroll 1
    for (;;) {
        const int cost = cost_of(s, q, w.p);
        if (rem < cost) break;
        rem -= cost;
        ++w.p;
    }
    w.j = static_cast<int>(rem);
    w.left = left;
    return w;
}
PREFIX_HD int64_t places_of(const Shape &s, const Seq &q, int *longest) {
    const int pairs = pairs_of(s, q);
    int64_t head = 0;
#pragma unroll 1
    for (int p = 0; p < pairs; ++p) {
        const int cost = cost_of(s, q, p);
        *longest = imax(*longest, cost);
        head += cost;
    }
    return head * s.heads;
}

// A call's workspace, as offsets from its base: the cuts, maximum and sum of the partial results' rows, their
// columns. Columns are written and read 32 bytes at a time, and the base is a multiple of 16 only: the layout
// begins on the next 32-byte bound, for which `bytes` has room whatever the base.
constexpr size_t kPartAlign = 32, kBaseAlign = 16;
struct Workspace {
    size_t cut, ml, o, bytes;
};
inline Workspace workspace_at(uintptr_t base, size_t cut_bytes, int columns) {
    const size_t slots = 2 * kMaxCtas * 2 * kRows;
    Workspace w;
    w.cut = (kPartAlign - base % kPartAlign) % kPartAlign;
    w.ml = w.cut + (cut_bytes * kMaxCtas + 255) / 256 * 256;
    w.o = w.ml + 2 * sizeof(float) * slots;
    w.bytes = w.o - w.cut + sizeof(float) * slots * columns + kPartAlign - kBaseAlign;
    return w;
}

}  // namespace tree
}  // namespace rps
