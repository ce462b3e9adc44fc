// prefix_attention.cu -- attention of the sequences' newest tokens over the paged
// K/V cache, the pages that the sequences of a request share read once for a tile of
// 128 query rows of all of them (rps_prefix_attention_fwd).
//
// For query i of a sequence, out = sum_j softmax_j(scale q . k_j) v_j over the keys
// it sees. The softmax over two sets of keys is joined from the sets' maxima m, sums
// l and weighted sums o: with m = max(m1, m2) both sides are weighted by
// 2^(m_x - m) and added. So the keys of a row may be taken in any pieces: the
// sequences of a request, and the query heads that share a cache head, are stacked
// as the 128 rows of one matrix product with the shared keys; their own keys follow
// as further key tiles of the same row tile, each 16-key step of the product
// writing only its sequence's rows; and the key tiles of all row tiles are dealt to
// the CTAs by equal costs (prefix_split.h), whose partial (m, l, o) a second launch joins.
//
// One persistent CTA per SM takes pieces (row tile, key tiles [j0, j1)). Key tiles
// are numbered through its pieces; even and odd ones go to two independent halves
// of the softmax, each with its own S / P buffer, maxima, sums and accumulator:
//   warp 0      TMA producer of K, one box per slot of pages, addresses through the
//               page table, and of Q (a box of tokens x heads of the group);
//   warp 2      TMA producer of V, in the same way. V lies token by token in the
//               cache, so it is the MN-major operand of the second product: no
//               transposed copy of the values is kept;
//   warp 3      cleaner of own tiles' V: clears the rows past a sequence's last key (they
//               may hold anything, and 0 * NaN would reach the sums), and lists which
//               rows each 16-key step of the product writes;
//   warp 1      MMA issuer, one thread: S = Q K^T into TMEM buffer t % 2, O[t % 2] += P V
//               with P from TMEM, in the order PV(t), S(t + 2), PV(t + 1), ...;
//   warps 4-7   softmax of even tiles, 8-11 of odd ones: thread = row. One pass with a
//               standing base-2 reference, which is changed only where a tile's sum is
//               far out of range. P is rounded to the cache's type (the product takes
//               no other); its sum is taken before the rounding, in fp32;
//   warps 12-15 read-out: the halves' accumulators weighted and added; written as
//               output rows, or as fp32 partial results where a piece is not all
//               of its row tile. Warp 12 also schedules: it finds the pieces from the
//               lengths in device memory and hands them to the other roles through a
//               ring in shared memory.
//
// What bounds it, at the figures measured (times of both launches):
//   2 requests, 28 / 4 heads, 9 branches of 32, contexts to 32700, fp16: 169 us, 1390
//     TFLOP/s. A key tile takes 1600 to 1690 cycles, of which MMAs execute in 1024: two tiles
//     take as long as the chain of one half (softmax 1730, P handed on 90, PV issued 150,
//     its commit and K's wait 420, S issued 220, S executed and seen 580). The clock is the
//     power limit's (1.45 to 1.9 GHz). Slower: two row tiles sharing K and V stages (195), two
//     issuing warps (240), unrolled batches (187), K awaited before the products (194).
//   64 requests, 32 heads, 9 branches of 32, contexts 200 to 1200 in pages of 16: 382
//     us, 3.5 TB/s of cache, queries and outputs. A row tile has 6 shared tiles and 1.6 own
//     ones: the change to the next takes 2800 cycles (the read-out hands O back after 1900;
//     half of O at once, in 128 registers, was slower), own tiles half as much again
//     as shared ones, and a stage of K is free only 2600 cycles before its next use, of which
//     the copies take 2200. Instruction fetches: 76 KB of code in all roles, 5 % of the
//     fetches miss the cache (158 KB missed 32 %).
//   One request's 9 branches of 32, 32 heads, context 328: 17 us; 64 sequences of one
//     prompt of 8200: 28. About 6 us pass before a CTA's first copy (lengths, prefix
//     sums, the range's begin, the page table: dependent accesses), 2 in the second launch.
// Every wait is bounded; a role whose wait runs out flags RPS_DEVERR_TIMEOUT and
// raises the CTA's abort flag, copies and MMAs in flight are drained and TMEM is
// freed before the CTA exits.
#include <cuda.h>  // CUtensorMap and the tensor-map encoder's signature (no link against the driver)
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>

#include "prefix_split.h"
#include "rps_internal.cuh"
#include "tc_device.cuh"
#include "umma_desc.h"

namespace rps {
namespace {

using prefix::kMaxCtas;
using prefix::KeySum;
using prefix::RowTile;
using prefix::Shape;
using prefix::Tiles;

constexpr int kD = 128;                // head dimension
constexpr int kAtom = 64 * 128 * 2;    // one 128-row x 64-column swizzle atom of 16-bit elements: 16 KB
constexpr int kTileBytes = 2 * kAtom;  // a Q, K or V tile: Q's two atoms along d
// A K or V tile goes in groups of 8 tokens: their columns 0..63, then 64..127 (1024 bytes each).
constexpr int kChunk = 1024, kGroup = 2 * kChunk;
constexpr int kStages = 2;             // of K and of V: a tile's stage, S / P buffer and O go by its parity
constexpr int kQBufs = 2;
constexpr int kStageBytes = 32 * 128;  // per read-out warp: 32 rows x 128 bytes on their way out
constexpr int kSmemBytes = kQBufs * kTileBytes + 2 * kStages * kTileBytes + 4 * kStageBytes + 1024;
constexpr int kThreads = 512;
// 128 x 56 + 256 x 144 + 128 x 168 = 65,536 registers of the 512 x 128 of the launch
constexpr int kCtlRegs = 56, kSoftRegs = 144, kOutRegs = 168;
static_assert(128 * kCtlRegs + 256 * kSoftRegs + 128 * kOutRegs <= 512 * 128, "the split fits the launch's registers");
constexpr uint32_t kTmemCols = 512;  // S buffers at columns 0 and 128, O at 256 and 384
constexpr uint32_t kOCol = 256;
constexpr int kRing = 4;             // pieces known ahead
constexpr int kConsumers = 16;       // every warp
constexpr int kMaxSeqs = 128;        // sequences with rows in one row tile
constexpr int kStepAdds = 32;
// Lengths, and key tiles of a head's row tiles (a block of threads' at most), are kept in shared
// memory where they fit (64 sequences of one prompt: 31 us instead of 33.7).
constexpr int kStagedLens = 512;
constexpr int kStagedTiles = 512;
constexpr uint32_t kNoEnd = 1u << 31;  // tiles of the CTA, until its last piece is known
constexpr int kMaxReqs = 2 * kStages * kTileBytes / 8;  // requests whose first costs fit the K and V stages
constexpr float kLn2 = 0.6931471805599453f;
// bounds of a tile's sum of P in a row (in units of its reference): P in fp16 stays finite
constexpr float kMostWeight = 32768.f, kLeastWeight = 1.f / 32768.f;

// A row tile that is cut: the CTA that takes its first key tile writes where its parts
// are, into the row tile's entry or its own (prefix::cut_list).
struct Cut {
    int32_t parts;       // 0: none
    int32_t cta;         // the first part's
    int32_t q, head, rt;
};

struct PrefixArgs {
    Shape s;
    const int32_t *table, *len, *shared_len;
    int32_t n_heads;  // query heads
    void *out;
    int64_t out_req, out_token, out_head;
    float *lse;
    float c;  // scale * log2(e)
    // A copy of K or V takes 2^copy_log tokens. by_groups: from a map whose third dimension goes
    // through the tokens of all pages by eights, page_groups of them a page; else 8 tokens of a page
    int32_t by_groups, copy_log, page_groups, no_page;  // no_page: a coordinate beyond the pages
    Cut *cut;       // [kMaxCtas]
    int32_t by_tile;  // cuts are listed by row tile
    float2 *part_ml;  // [2 * kMaxCtas][128]: maximum and sum of each row of a partial result
    float *part_o;    // [2 * kMaxCtas][128][128]
    uint32_t *err;
    uint32_t tries;  // of a wait
};

struct Piece {
    int32_t q, head, rt;
    RowTile r;
    int32_t j0, j1, shared, shared_tiles, shared_row;  // shared slots; whose table row names their pages
    int32_t part;                                      // -1: the whole row tile, else which partial result
    int32_t last;                                      // of the CTA
    int32_t off[kMaxSeqs + 1], len[kMaxSeqs];
};

struct Ctl {
    // s_full[t % 2]: S of tile t is computed and the product of tile t - 2 is done, so
    // K stage t % 2 is free, and Q of the pieces before t's. V stages have a commit of
    // their own. No wait sees a barrier two phases on: each waits for every phase in turn.
    uint64_t q_full[kQBufs], k_full[kStages], v_full[kStages], v_empty[kStages], v_raw[kStages];
    uint64_t s_full[kStages], p_full[kStages], o_ready, o_free, mma_done;
    uint64_t ring_full[kRing], ring_empty[kRing];
    // a half's reference and sum of a row at the end of piece n, in slot n % 4: written before
    // the half's last P of the piece is handed on, read once O is ready, and written again for
    // piece n + 4, whose P needs the products of piece n + 2 and so the read-out of piece n + 1
    float2 ml[4][kStages][prefix::kRows];
    Piece ring[kRing];
    // own tile in V stage s, from V's cleaner: rows that step kk leaves alone; its keys (0: no
    // step), and kStepAdds unless it overwrites
    uint4 step_off[kStages][8];
    int32_t step_how[kStages][8];
    int4 copy_at[2][32];  // a producer's copies: their coordinates, of two tiles
    uint32_t bad[4];  // copies of key tile t whose page id is outside the cache (t % 4)
    int64_t scan[16];
    int32_t len[kStagedLens];      // as they are used
    int32_t longest, empty;  // cost of the most expensive row tile; one has no key tile
    uint32_t tmem_base;
    int abort_flag;
};

// ---------------------------------------------------------------- waits
// One try of a wait for a phase, which the hardware suspends for about a microsecond at most.
__device__ __forceinline__ bool try_wait_us(uint64_t *bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(saddr(bar)), "r"(parity), "r"(1000u)
        : "memory");
    return done != 0;
}
// Waits for a phase of a barrier, at most a.tries tries, all lanes; the warp goes on
// together, on the same answer. A wait that runs out raises the abort flag, which is
// reported when the CTA ends; the other roles' waits then run out too. (Short: every role's
// waits are inlined, and the roles' code has to fit the instruction cache together.)
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, Ctl &c, const PrefixArgs &a) {
    bool ok = false;
#pragma unroll 1
    for (uint32_t i = 0; i < a.tries && !ok; ++i) ok = try_wait_us(bar, parity);
    if (__all_sync(kFull, ok)) return true;
    *reinterpret_cast<volatile int *>(&c.abort_flag) = 1;
    return false;
}

// One thread of the converged warp, known to the compiler as one.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
// Waits for what is in flight when a role ends, a fifth of a second at most.
__device__ __forceinline__ void drain(uint64_t *bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t i = 0; i < 200000 && !try_wait_us(bar, parity); ++i) {
    }
}

// ---------------------------------------------------------------- the cut
__device__ __forceinline__ int len_of(const PrefixArgs &a, int s, const Ctl &c) {
    return a.s.n_req * a.s.n_branch <= kStagedLens ? c.len[s] : prefix::used_len(a.s, a.len[s]);
}
__device__ __forceinline__ int shared_len_of(const PrefixArgs &a, int q) { return a.shared_len ? a.shared_len[q] : 0; }

// Key tiles of row tile rt of request q, by one thread.
__device__ __forceinline__ Tiles entry_tiles(const PrefixArgs &a, int q, int rt, int shared_len, const Ctl &c) {
    const RowTile r = prefix::row_tile(a.s, rt);
    KeySum k{0, 0, INT32_MAX};
    const int s0 = q * a.s.n_branch + r.b0;
    if (a.s.n_req * a.s.n_branch <= kStagedLens) {
#pragma unroll 4
        for (int i = 0; i < r.nb; ++i) prefix::add_sequence(a.s, k, c.len[s0 + i]);
    } else {
#pragma unroll 1
        for (int i = 0; i < r.nb; ++i) prefix::add_sequence(a.s, k, prefix::used_len(a.s, a.len[s0 + i]));
    }
    return prefix::key_tiles(a.s, k, prefix::shared_slots(a.s, k, shared_len));
}
// What find_range leaves for find_start, in the buffers of Q, K and V, which nothing uses before the
// first piece is known.
struct Plan {
    int64_t *first;  // costs (of one head: all heads of a request have the same) of the requests before q
    Tiles *tiles;    // of (request, row tile), where they are kept
};
__device__ __forceinline__ Tiles known_tiles(const PrefixArgs &a, int q, int rt, const Plan &plan, const Ctl &c) {
    return a.s.n_req * a.s.row_tiles <= kStagedTiles ? plan.tiles[q * a.s.row_tiles + rt]
                                                     : entry_tiles(a, q, rt, shared_len_of(a, q), c);
}

// Exclusive prefix sum over the block's 512 threads; *total: the block's sum.
__device__ __forceinline__ int64_t scan_block(int v, int64_t *sums, int64_t *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(kFull, x, o);
        if (lane >= o) x += u;
    }
    __syncthreads();  // (the sums of an earlier scan are read)
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += sums[w];
        all += sums[w];
    }
    *total = all;
    return before + x - v;
}

// The CTA's range of the costs of all (request, head, row tile) in order (at == end: it has
// nothing to do); or (whole) its one row tile.
struct Range {
    int64_t at, end;
    prefix::Ranges all;
    bool whole;
};
// Cutting a row tile costs what its parts take to be written and joined, about as much as
// three own tiles: where every row tile has a CTA of its own and none costs by more than
// that more than the equal shares, none is cut (one request's 9 branches of 32, 32 heads, context
// 328: 96 row tiles of 4 to 5 key tiles instead of shares of 3: 17 us instead of 21; one query of 32
// heads over 1000 keys, which are worth cutting: 18 instead of 19.6).
constexpr int kCutCost = 3 * prefix::kOwnCost;

// By all threads: the lengths into shared memory, and the plan.
__device__ __forceinline__ Range find_range(const PrefixArgs &a, Ctl &c, const Plan &plan) {
    const int entries = a.s.n_req * a.s.row_tiles, n_seq = a.s.n_req * a.s.n_branch;
    if (n_seq <= kStagedLens)
#pragma unroll 1
        for (int i = threadIdx.x; i < n_seq; i += kThreads) c.len[i] = prefix::used_len(a.s, a.len[i]);
    if (threadIdx.x == 0) c.longest = c.empty = 0;
    // (loaded while the lengths are)
    int next_shared = shared_len_of(a, min(prefix::quotient(threadIdx.x, a.s.by_row_tiles), a.s.n_req - 1));
    __syncthreads();
    const bool few = static_cast<int64_t>(entries) * a.s.heads <= gridDim.x;  // (at most one block of entries then)
    int64_t carry = 0;
#pragma unroll 1
    for (int base = 0; base < entries; base += kThreads) {
        const int e = base + threadIdx.x;
        const int q = prefix::quotient(e, a.s.by_row_tiles), rt = e - q * a.s.row_tiles;
        int64_t total;
        Tiles t{0, 0};
        if (e < entries) t = entry_tiles(a, q, rt, next_shared, c);
        const int cost = prefix::cost_of(t);
        if (entries <= kStagedTiles && e < entries) plan.tiles[e] = t;
        if (base + kThreads < entries)
            next_shared = shared_len_of(a, min(prefix::quotient(e + kThreads, a.s.by_row_tiles), a.s.n_req - 1));
        if (few && e < entries) {
            if (cost == 0) c.empty = 1;
            atomicMax(&c.longest, cost);
        }
        const int64_t before = carry + scan_block(cost, c.scan, &total);
        if (e < entries && rt == 0) plan.first[q] = before;
        carry += total;
    }
    Range r{};
    const int64_t work = carry * a.s.heads;
    // (no more CTAs than have a tile each: none in between is without work)
    const int64_t most = work / prefix::kWidest;
    const int n = static_cast<int>(min(static_cast<int64_t>(gridDim.x), most > 0 ? most : static_cast<int64_t>(work > 0)));
    if (few && !c.empty && static_cast<int64_t>(c.longest - kCutCost) * n <= work) {
        r.whole = true;
        r.end = static_cast<int>(blockIdx.x) < entries * a.s.heads ? 1 : 0;
        return r;
    }
    if (static_cast<int>(blockIdx.x) >= n) return r;
    r.all = prefix::make_ranges(work, n);
    r.at = prefix::range_start(r.all, blockIdx.x);
    r.end = prefix::range_start(r.all, blockIdx.x + 1);
    return r;
}

// By a warp: the request, head, row tile and key tile that the range begins with.
struct Start {
    int32_t q, head, rt, j;  // (j past the row tile's last tile: the range begins with the next row tile)
    int64_t base;            // costs before the row tile
    Tiles tiles, next;       // of the row tile and of the next of the head (none, or not known: 0)
};
__device__ __forceinline__ Start find_start(const PrefixArgs &a, const Range &range, const Plan &plan, int lane,
                                            const Ctl &c) {
    Start st{};
    if (range.whole) {
        const int qh = prefix::quotient(blockIdx.x, a.s.by_row_tiles);
        st.rt = blockIdx.x - qh * a.s.row_tiles;
        st.q = qh / a.s.heads;
        st.head = qh - st.q * a.s.heads;
        return st;
    }
    int lo = 0, hi = a.s.n_req;  // the last request that starts at or before the range
#pragma unroll 1
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (plan.first[mid] * a.s.heads <= range.at)
            lo = mid;
        else
            hi = mid;
    }
    st.q = lo;
    int64_t rem = range.at - plan.first[lo] * a.s.heads;  // cost of the request before the range
    int64_t per_head = 0;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {  // the cost of a head; then where the rest lies in it
        int64_t before = 0;
#pragma unroll 1
        for (int base = 0; base < a.s.row_tiles; base += 32) {
            Tiles t{0, 0};
            if (base + lane < a.s.row_tiles) t = known_tiles(a, st.q, base + lane, plan, c);
            const int cost = prefix::cost_of(t);
            int upto = cost;
#pragma unroll 1
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(kFull, upto, o);
                if (lane >= o) upto += u;
            }
            if (pass == 1) {
                const uint32_t in = __ballot_sync(kFull, rem < before + upto);
                if (in) {
                    const int who = __ffs(in) - 1;
                    const int64_t y = rem - before - __shfl_sync(kFull, upto - cost, who);
                    st.rt = base + who;
                    st.tiles.shared = __shfl_sync(kFull, t.shared, who);
                    st.tiles.own = __shfl_sync(kFull, t.own, who);
                    st.next.shared = __shfl_sync(kFull, t.shared, (who + 1) & 31);
                    st.next.own = __shfl_sync(kFull, t.own, (who + 1) & 31);
                    if (who == 31) st.next.shared = st.next.own = 0;
                    st.j = prefix::reach(st.tiles, y);
                    st.base = range.at - y;
                    break;
                }
            }
            before += __shfl_sync(kFull, upto, 31);
        }
        if (pass == 0) {
            per_head = before;
            lo = 0, hi = a.s.heads;
#pragma unroll 1
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (mid * per_head <= rem)
                    lo = mid;
                else
                    hi = mid;
            }
            st.head = lo;
            rem -= lo * per_head;
        }
    }
    return st;
}

// Row tile rt of request q, by a warp: sequences' lengths and own slots into `p`;
// returns its key tiles (none: no sequence there, `p` is not complete).
__device__ __forceinline__ Tiles fill_row_tile(const PrefixArgs &a, int q, int rt, int lane, const Ctl &c, Piece &p) {
    const RowTile r = prefix::row_tile(a.s, rt);
    const int s0 = q * a.s.n_branch + r.b0;
    KeySum k{0, 0, INT32_MAX};
    int first = INT32_MAX;
    const int shared_len = shared_len_of(a, q);
#pragma unroll 1
    for (int i = lane; i < r.nb; i += 32) {
        const int len = len_of(a, s0 + i, c);
        p.len[i] = len;
        prefix::add_sequence(a.s, k, len);
        if (len >= 0) first = min(first, i);
    }
    k.present = __reduce_add_sync(kFull, k.present);
    k.slots = __reduce_add_sync(kFull, k.slots);
    k.min_pages = __reduce_min_sync(kFull, k.min_pages);
    first = __reduce_min_sync(kFull, first);
    const int shared = prefix::shared_slots(a.s, k, shared_len);
    const Tiles tiles = prefix::key_tiles(a.s, k, shared);
    if (!k.present) return tiles;
    int before = 0;
#pragma unroll 1
    for (int base = 0; base < r.nb; base += 32) {
        const int i = base + lane, len = i < r.nb ? p.len[i] : -1;
        const int own = len < 0 ? 0 : prefix::slots_of(a.s, len) - shared;
        int upto = own;
#pragma unroll 1
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(kFull, upto, o);
            if (lane >= o) upto += u;
        }
        if (i < r.nb) p.off[i + 1] = before + upto;
        before += __shfl_sync(kFull, upto, 31);
    }
    if (lane == 0) {
        p.off[0] = 0;
        p.q = q;
        p.rt = rt;
        p.r = r;
        p.shared = shared;
        p.shared_tiles = tiles.shared;
        p.shared_row = s0 + first;
    }
    return tiles;
}

// ---------------------------------------------------------------- roles
// Piece n of the CTA, once the scheduler has it (nullptr: the wait ran out).
__device__ __forceinline__ const Piece *next_piece(int n, Ctl &c, const PrefixArgs &a) {
    if (!warp_wait(&c.ring_full[n % kRing], (n / kRing) & 1, c, a)) return nullptr;
    return &c.ring[n % kRing];
}
__device__ __forceinline__ void release_piece(int n, int lane, Ctl &c) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&c.ring_empty[n % kRing]);
}

// The page id (as the table has it: the load is on its way) of copy `lane` of key tile j and the
// copy's first token in the page; false: the tile has no such copy.
__device__ __forceinline__ bool copy_page(const PrefixArgs &a, const Piece &p, int j, int lane, int2 &at) {
    const int log = a.s.slot_log - a.copy_log;  // copies of a slot
    const bool own = j >= p.shared_tiles;
    int row = p.shared_row, x = ((own ? j - p.shared_tiles : j) << a.s.spt_log) + (lane >> log);
    if (lane >> log >= a.s.spt || x >= (own ? p.off[p.r.nb] : p.shared)) return false;
    if (own) {
        const int i = prefix::slot_owner(p.off, p.r.nb, x);
        x += p.shared - p.off[i];
        row = p.q * a.s.n_branch + p.r.b0 + i;
    }
    at = make_int2(a.table[static_cast<int64_t>(row) * a.s.max_pages + (x >> a.s.sub_log)],
                   ((x & (a.s.sub - 1)) << a.s.slot_log) + ((lane & ((1 << log) - 1)) << a.copy_log));
    return true;
}

// One thread's wait.
__device__ __forceinline__ bool lane_wait(uint64_t *bar, uint32_t parity, Ctl &c, const PrefixArgs &a) {
#pragma unroll 1
    for (uint32_t i = 0; i < a.tries; ++i)
        if (try_wait_us(bar, parity)) return true;
    *reinterpret_cast<volatile int *>(&c.abort_flag) = 1;
    return false;
}

// The producers of K (with Q) and of V, in one body: two warps run it.
__device__ __forceinline__ void produce(bool is_k, const CUtensorMap *tm, const CUtensorMap *tm_q, uint8_t *stages,
                                        uint8_t *sq, uint32_t tiles, int lane, Ctl &c, const PrefixArgs &a) {
    uint32_t t = 0;
    int n = 0, n_q = 0, raw0 = 0, raw1 = 0;  // V tiles of each stage that went to v_raw
    uint32_t raw_last = 0;                   // bit s: the last of stage s did
    bool ok = true;
    uint64_t *full = is_k ? c.k_full : c.v_full;
    // K: S of tile t - 2 is computed, so its stage is free, and at a piece's first tile the Q
    // buffer of piece n - 2, whose last tile is no later. V: the product of tile t - 2 is done.
    uint64_t *empty = is_k ? c.s_full : c.v_empty;
#pragma unroll 1
    for (; t < tiles && ok; ++n) {
        const Piece *pp = next_piece(n, c, a);
        if (!pp) break;
        const Piece &p = *pp;
        if (p.last) tiles = t + p.j1 - p.j0;
#pragma unroll 1
        for (int j = p.j0; ok && j < p.j1; j += 2) {
            // two tiles are looked up at a time, half a warp each: with votes and shared memory it takes as
            // long as a tile's copies (64 requests, contexts 200 to 1200: 387 us with one, 382 with two)
            const int two = min(2, p.j1 - j), half = lane >> 4;
            int2 at = make_int2(-1, 0);
            const bool there = half < two && copy_page(a, p, j + half, lane & 15, at);
            // (an id outside the cache: a coordinate whose copy is all zeros, as are copies that are not there)
            const bool bad_page = static_cast<unsigned>(at.x) >= static_cast<unsigned>(a.s.n_pages);
            c.copy_at[is_k][lane] =
                a.by_groups ? make_int4(0, bad_page ? a.no_page : at.x * a.page_groups + (at.y >> 3), p.head, 0)
                            : make_int4(at.y, p.head, bad_page ? a.no_page : at.x, 0);
            const uint32_t bad = __ballot_sync(kFull, there && bad_page);
            if (bad && is_k && lane == 0) flag_error(a.err, RPS_DEVERR_PAGE);
            __syncwarp();
            int done = 0;
            if (elect_one()) {
#pragma unroll 1
                for (; done < two; ++done) {
                    const uint32_t x = t + done;
                    const int s = x % kStages;
                    if (x >= kStages && !lane_wait(&empty[s], (x / kStages - 1) & 1, c, a)) break;
                    // (V of own tiles goes through the cleaner)
                    uint64_t *bar = !is_k && j + done >= p.shared_tiles ? &c.v_raw[s] : &full[s];
                    // (before the arrival, which hands it on to the softmax of tile x; that of tile x - 4 has read its own)
                    if (is_k) c.bad[x % 4] = bad >> done * 16 & 0xffffu;
                    mbar_expect_tx(bar, kTileBytes);
                    // (coordinates from shared memory: picked out of lanes a copy took a third longer)
                    uint8_t *dst = stages + s * kTileBytes;
                    const int4 *from = &c.copy_at[is_k][done * 16];
                    int4 at = from[0];
#pragma unroll 1
                    for (int i = 1; i <= prefix::kRows >> a.copy_log; ++i, dst += kGroup / 8 << a.copy_log) {
                        const int4 next = from[i & 15];
                        tma_load_5d(dst, tm, 0, at.x, 0, at.y, at.z, bar);
                        at = next;
                    }
                    if (is_k && j + done == p.j0) {  // Q: its buffer's last user, piece n - 2, ended at tile x - 2 or before
                        uint64_t *q_full = &c.q_full[n & 1];
                        mbar_expect_tx(q_full, 2u * a.s.group * a.s.tokens * 128);
                        dst = sq + (n & 1) * kTileBytes;
                        tma_load_4d(dst, tm_q, 0, p.head * a.s.group, p.r.tok0, p.q, q_full);
                        tma_load_4d(dst + kAtom, tm_q, 64, p.head * a.s.group, p.r.tok0, p.q, q_full);
                    }
                }
            }
            done = __reduce_max_sync(kFull, done);
            ok = done == two;
            n_q += is_k && j == p.j0 && done > 0;
#pragma unroll 1
            for (int u = 0; u < done; ++u, ++t) {
                const int s = t % kStages;
                const bool raw = !is_k && j + u >= p.shared_tiles;
                raw_last = (raw_last & ~(1u << s)) | (raw ? 1u << s : 0u);
                raw0 += raw && s == 0;
                raw1 += raw && s == 1;
            }
        }
        if (ok) release_piece(n, lane, c);
    }
    // every copy issued lands before the CTA leaves
    if (lane == 0) {
#pragma unroll 1
        for (uint32_t x = t > kStages ? t - kStages : 0; x < t; ++x) {
            const int s = x % kStages;
            if (raw_last >> s & 1u)
                drain(&c.v_raw[s], ((s ? raw1 : raw0) - 1) & 1);
            else
                drain(&full[s], (x / kStages) & 1);
        }
#pragma unroll 1
        for (int x = n_q > kQBufs ? n_q - kQBufs : 0; x < n_q; ++x) drain(&c.q_full[x & 1], (x >> 1) & 1);
    }
    __syncwarp();
}

// The cleaner of V, for own tiles: prepares the product's steps, and clears the rows of V past a
// sequence's last key before the product may read the tile (they may hold anything, and 0 * NaN
// would be added). A warp of its own, for the producer has the next tile's copies to issue meanwhile.
__device__ __forceinline__ void clean(uint8_t *stages, uint32_t tiles, int lane, Ctl &c, const PrefixArgs &a) {
    uint32_t t0 = 0;
    int raw0 = 0, raw1 = 0;
#pragma unroll 1
    for (int n = 0; t0 < tiles; ++n) {
        const Piece *pp = next_piece(n, c, a);
        if (!pp) return;
        const Piece &p = *pp;
        if (p.last) tiles = t0 + p.j1 - p.j0;
#pragma unroll 1
        for (int j = max(p.j0, p.shared_tiles); j < p.j1; ++j) {
            const int s = (t0 + j - p.j0) % kStages;
            const prefix::Step st = prefix::own_step(a.s, p.r, p.off, p.len, p.shared_tiles, p.shared, p.j0, j, lane & 7);
            const int keys = lane < 8 ? st.keys : 0;
            // (the stage's copies were issued once the product before had read its steps)
            if (!warp_wait(&c.v_raw[s], (s ? raw1 : raw0) & 1, c, a)) return;
            raw0 += s == 0;
            raw1 += s;
            if (lane < 8) {
                c.step_off[s][lane] = make_uint4(
                    ~(low_bits(st.r1) & ~low_bits(st.r0)), ~(low_bits(st.r1 - 32) & ~low_bits(st.r0 - 32)),
                    ~(low_bits(st.r1 - 64) & ~low_bits(st.r0 - 64)), ~(low_bits(st.r1 - 96) & ~low_bits(st.r0 - 96)));
                c.step_how[s][lane] = keys > 0 ? keys | (st.fresh ? 0 : kStepAdds) : 0;
            }
            uint8_t *vb = stages + s * kTileBytes;
#pragma unroll 1
            for (uint32_t m = __ballot_sync(kFull, keys > 0 && keys < 16); m; m &= m - 1) {
                const int kk = __ffs(m) - 1, filled = __shfl_sync(kFull, keys, kk);
#pragma unroll 1
                for (int y = lane; y < (16 - filled) * 16; y += 32) {  // 8 16-byte units in each of two chunks
                    const int token = kk * 16 + filled + (y >> 4);
                    st_shared_v4(saddr(vb + token / 8 * kGroup + (y & 8 ? kChunk : 0) + token % 8 * 128 + (y & 7) * 16),
                                 make_uint4(0, 0, 0, 0));
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.v_full[s]);
        }
        t0 += p.j1 - p.j0;
        release_piece(n, lane, c);
    }
}

// The scheduler: one warp hands out the pieces of the CTA's range, one per call.
struct Schedule {
    Start st;
    int q, head, rt, j, n;
    int64_t base, end;       // costs before the row tile, and the range's end
    int cost;                // of the row tile
    bool swapped, any, done; // swapped: the second of two row tiles comes first; any: the request has a key tile at all
    bool leave;              // the row tile, at the next call
};

__device__ __forceinline__ Schedule schedule_start(const PrefixArgs &a, const Range &range, const Plan &plan, int lane,
                                                   Ctl &c) {
    Schedule z;
    z.st = find_start(a, range, plan, lane, c);
    // (the plan lies where Q, K and V go: the copies that follow the first piece come after its reads)
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    z.q = z.st.q;
    z.head = z.st.head;
    z.rt = z.st.rt;
    z.j = z.st.j;
    z.n = 0;
    z.base = z.st.base;
    z.end = range.end;
    z.cost = 0;
    z.swapped = z.leave = false;
    z.any = true;
    z.done = range.at == range.end;
    // A range that ends one row tile and begins the next of the same head is taken in the
    // other order: all CTAs of the head are then near the same keys at the same time,
    // which L2 holds, instead of all over them (2 requests, 28/4 heads, context 28000: the keys
    // were read from HBM seven times).
    const Tiles &t = z.st.tiles, &next = z.st.next;
    if (z.j > 0 && z.j < t.shared + t.own) {
        const int64_t after = z.base + prefix::cost_of(t);
        const int rest = prefix::reach(next, z.end - after);
        if (rest > 0 && rest < next.shared + next.own) {
            z.swapped = true;
            z.base = after;
            ++z.rt;
            z.j = 0;
        }
    }
    return z;
}

// The next piece into the ring; false: there is none, or the wait for its slot ran out.
__device__ __forceinline__ bool schedule_next(Schedule &z, const PrefixArgs &a, const Range &range, int lane, Ctl &c) {
    if (z.done) return false;
    const int slot = z.n % kRing;
    if (z.n >= kRing && !warp_wait(&c.ring_empty[slot], (z.n / kRing - 1) & 1, c, a)) return false;
    Piece &p = c.ring[slot];
    Tiles t;
    int tiles;
#pragma unroll 1
    for (;;) {
        if (z.leave) {
            z.base += z.cost;
            z.j = 0;
            if (++z.rt == a.s.row_tiles) {
                z.rt = 0;
                if (!z.any || ++z.head == a.s.heads) {
                    z.head = 0;
                    ++z.q;
                }
                z.any = false;
            }
        }
        z.done = z.q >= a.s.n_req;  // (not reached while the lengths stay as they are during the call)
        if (z.done) return false;
        z.leave = true;
        t = fill_row_tile(a, z.q, z.rt, lane, c, p);
        z.cost = prefix::cost_of(t);
        tiles = t.shared + t.own;
        z.any |= tiles > 0;
        if (tiles > z.j) break;
    }
    const int64_t left = z.end - z.base;  // of the range, from the row tile's begin
    const int j1 = range.whole ? tiles : prefix::reach(t, left);
    const bool first_of_two = z.swapped && z.rt != z.st.rt;
    const bool last = !first_of_two && (range.whole || z.swapped || left - z.cost < prefix::kFirstPlace);
    z.done = last || j1 <= z.j;
    if (j1 <= z.j) return false;  // (nor this)
    if (lane == 0) {
        p.head = z.head;
        p.j0 = z.j;
        p.j1 = j1;
        p.part = z.j == 0 && j1 == tiles ? -1 : z.j > 0 ? 0 : 1;
        p.last = last;
        const int tile = (z.q * a.s.heads + z.head) * a.s.row_tiles + z.rt;
        if (p.part == 1) {
            const int to = prefix::cta_of(range.all, z.base + prefix::place(t, tiles - 1) - 1);
            a.cut[a.by_tile ? tile : static_cast<int>(blockIdx.x)] =
                Cut{to - static_cast<int>(blockIdx.x) + 1, static_cast<int>(blockIdx.x), z.q, z.head, z.rt};
        } else if (p.part < 0 && a.by_tile) {
            a.cut[tile].parts = 0;
        }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&c.ring_full[slot]);
    ++z.n;
    if (first_of_two) {
        z.rt = z.st.rt;
        z.j = z.st.j;
        z.base = z.st.base;
        z.leave = false;
    }
    return true;
}

// The MMA issuer, one thread: S_t = Q K_t^T into TMEM buffer t % 2, O[t % 2] += P_t V_t. The tensor
// pipe runs them in order, so S of tile t + 2 may overwrite the P that the product of tile t
// reads without a wait. An issued instruction holds the thread until the pipe takes it, and
// what the thread does between the batches leaves the pipe idle: so there is one wait for each
// batch, and one thread without votes, elected (so the compiler knows that it is alone and keeps the
// operands in uniform registers: 353 -> 341 us against lane 0, 64 requests, context 704).
template <bool kF16>
__device__ __forceinline__ void issue_products(uint8_t *sq, uint8_t *sk, uint8_t *sv, uint32_t tmem, uint32_t tiles,
                                               int lane, Ctl &c, const PrefixArgs &a) {
    if (elect_one()) {
        constexpr uint32_t fmt = kF16 ? umma::kFmtF16 : umma::kFmtBF16;
        constexpr uint32_t idesc_s = umma::instr_desc_f16(128, 128, fmt, 0);  // K is K-major
        constexpr uint32_t idesc_o = umma::instr_desc_f16(128, 128, fmt, 1);  // V is MN-major
        // (an operand's other buffer, atom or step: its address field moved on)
        const uint64_t q_desc = umma::smem_desc_kmajor_sw128(saddr(sq));
        const uint64_t k_desc = umma::smem_desc_kmajor_sw128(saddr(sk), kGroup);
        const uint64_t v_desc = umma::smem_desc_mnmajor_sw128(saddr(sv), kChunk, kGroup);
        int sn = -1, s_left = 0;                        // the scores' piece, and its tiles left
        int n = -1, j = 0, j0 = 0, j1 = 0, shared_tiles = 0;  // the product's piece and tile
        bool s_more = tiles > 0, s_last = false, last = false;
#pragma unroll 1
        for (uint32_t x = 0; tiles; ++x) {  // the product of tile x - 2, then the scores of tile x
            const uint32_t h = x % kStages, parity = (x / kStages) & 1;
            if (x >= kStages) {
                if (j == j1) {
                    if (n >= 0) mbar_arrive(&c.ring_empty[n % kRing]);
                    if (last) break;
                    ++n;
                    const Piece &p = c.ring[n % kRing];
                    // the first product of a piece overwrites O: the previous piece's read-out must be done
                    if (!lane_wait(&c.ring_full[n % kRing], (n / kRing) & 1, c, a) ||
                        !lane_wait(&c.o_free, (n & 1) ^ 1, c, a))
                        break;
                    j = j0 = p.j0;
                    j1 = p.j1;
                    shared_tiles = p.shared_tiles;
                    last = p.last;
                }
                if (!lane_wait(&c.p_full[h], parity ^ 1, c, a)) break;  // P, and V (see the softmax)
                tc_fence_after();
                // P of keys 16k..16k+15: 8 columns; those of keys 64.. begin where their scores did
                const uint32_t pcol = tmem + h * 128, ocol = pcol + kOCol;
                const uint64_t vd = v_desc + h * (kTileBytes >> 4);
                if (j < shared_tiles) {
                    const uint32_t more = j - j0 >= kStages;  // the half has had a tile of this piece
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        mma_ts(ocol, pcol + k / 4 * 64 + k % 4 * 8, vd + static_cast<uint64_t>(k * (2 * kGroup >> 4)), idesc_o,
                               k ? 1u : more);
                } else {
#pragma unroll 2
                    for (int k = 0; k < 8; ++k) {
                        const uint4 o = c.step_off[h][k];
                        const int how = c.step_how[h][k];
                        const uint32_t off[4] = {o.x, o.y, o.z, o.w};
                        if (how)
                            mma_ts_rows(ocol, pcol + k / 4 * 64 + k % 4 * 8, vd + static_cast<uint64_t>(k) * (2 * kGroup >> 4),
                                        idesc_o, off, how & kStepAdds);
                    }
                }
                commit(&c.v_empty[h]);
                if (++j == j1) commit(&c.o_ready);  // the piece's O is complete
            }
            if (s_more) {
                if (s_left == 0) {
                    ++sn;
                    if (!lane_wait(&c.ring_full[sn % kRing], (sn / kRing) & 1, c, a) ||
                        !lane_wait(&c.q_full[sn & 1], (sn >> 1) & 1, c, a))
                        break;
                    s_left = c.ring[sn % kRing].j1 - c.ring[sn % kRing].j0;
                    s_last = c.ring[sn % kRing].last;
                }
                if (!lane_wait(&c.k_full[h], parity, c, a)) break;
                tc_fence_after();
                const uint64_t qd = q_desc + (sn & 1 ? kTileBytes >> 4 : 0), kd = k_desc + h * (kTileBytes >> 4);
#pragma unroll
                for (int k = 0; k < 8; ++k)  // (16 of the 64 columns of an atom are 32 bytes)
                    mma_ss(tmem + h * 128, qd + k / 4 * (kAtom >> 4) + k % 4 * 2, kd + k / 4 * (kChunk >> 4) + k % 4 * 2,
                           idesc_s, k != 0);
                commit(&c.s_full[h]);
                if (--s_left == 0 && s_last) s_more = false;
            }
        }
        commit(&c.mma_done);
        drain(&c.mma_done, 0);
    }
    __syncwarp();
}

// Softmax of the tiles of half h; this thread's row is TMEM lane r.
template <bool kF16>
__device__ __forceinline__ void softmax(uint32_t tmem, int q, int lane, int h, uint32_t tiles, Ctl &c,
                                        const PrefixArgs &a) {
    const int r = q * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(q * 32) << 16;
    const uint32_t sbuf = tmem + lane_off + h * 128, obuf = tmem + lane_off + kOCol + h * 128;
    const int tok = prefix::quotient(r, a.s.by_group);  // the row's token in the tile
    bool ok = true;
    uint32_t t0 = 0;  // first tile of the piece
    for (int n = 0; t0 < tiles && ok; ++n) {
        const Piece *pp = next_piece(n, c, a);
        if (!pp) break;
        const Piece &p = *pp;
        int limit = 0, own_off = 0, own_end = 0;
        bool live = false;
        if (tok < p.r.n_tok) {
            const int g = p.r.tok0 + tok, b = prefix::quotient(g, a.s.by_n_q), i = b - p.r.b0;
            live = p.len[i] >= 0;
            limit = prefix::row_limit(a.s, p.len[i], g - b * a.s.n_q);
            own_off = p.off[i];
            own_end = p.off[i + 1];
        }
        float m = kF16 ? -INFINITY : 0.f, l = 0.f;
        const int count = p.j1 - p.j0, x0 = (h ^ static_cast<int>(t0)) & 1;
        if (p.last) tiles = t0 + count;
        for (int x = x0; x < count; x += kStages) {
            const uint32_t t = t0 + x;
            const int j = p.j0 + x;
            prefix::Columns col = prefix::row_columns(a.s, j, p.shared_tiles, p.shared, own_off, limit);
            if (!warp_wait(&c.s_full[h], (t / kStages) & 1, c, a)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t bad = c.bad[t % 4];
            if (bad && col.lo < col.hi) {  // a page of this row's keys does not exist: NaN
                const int u0 = col.lo >> a.copy_log, u1 = (col.hi - 1) >> a.copy_log;
                if (bad >> u0 & low_bits(u1 - u0 + 1)) {
                    l = NAN;
                    col.hi = col.lo;
                }
            }
            // A warp without a row whose P is read has nothing to do: steps of own tiles write the rows
            // of their sequence only, and what becomes of rows that are not stored does not matter.
            const int first = (j - p.shared_tiles) << a.s.spt_log;
            const bool takes = live && (j < p.shared_tiles || (own_off < first + a.s.spt && own_end > first));
            if (__any_sync(kFull, takes)) {
                // Keys that a row does not see take no weight: quarters (32 columns) in which some
                // row of the warp has such keys are masked and written back. (Rows that are not
                // stored need no mask: with 7 heads a group, two of every tile.)
                const bool part = live && (col.lo > 0 || col.hi < 128);
                if (__any_sync(kFull, part)) {
#pragma unroll 1
                    for (int k = 0; k < 128; k += 32) {
                        const int lo = part ? col.lo - k : 0, hi = part ? col.hi - k : 32;
                        if (!__any_sync(kFull, lo > 0 || hi < 32)) continue;
                        uint32_t s0[32];
                        tmem_ld32_async(sbuf + k, s0);
                        tmem_wait_dep(s0);
                        mask_scores(s0, lo, hi);
                        tmem_st32_u(sbuf + k, s0);
                    }
                    tmem_wait_st();
                }
                // P = 2^(s c - m) with the row's present reference m, 0 at first; the sum tells whether m
                // was good enough (P and the sums far from the ends of their types' ranges: for fp16
                // P, m is within 2^15 of the largest so far). If not, m becomes the tile's largest
                // score and P is computed again: P is kept in registers until then, for it overwrites scores.
                const f2 cc = pack2(a.c, a.c);
                bool raise = kF16 && m == -INFINITY && col.lo < col.hi;
#pragma unroll 1
                for (int round = 0; round < 2; ++round) {
                    if (__any_sync(kFull, raise)) {
                        float mx8[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) mx8[i] = -INFINITY;
#pragma unroll 1
                        for (int k = 0; k < 128; k += 32) {
                            uint32_t s0[32];
                            tmem_ld32_async(sbuf + k, s0);
                            tmem_wait_dep(s0);
                            max_scores(s0, mx8);
                        }
                        const float tm = fmaxf(fmaxf(fmaxf(mx8[0], mx8[1]), fmaxf(mx8[2], mx8[3])),
                                               fmaxf(fmaxf(mx8[4], mx8[5]), fmaxf(mx8[6], mx8[7]))) * a.c;
                        raise = raise && tm > -INFINITY;
                        const float f = raise && l != 0.f ? ex2(m - tm) : 1.f;  // (without weight so far: O is 0)
                        if (raise) m = tm;
                        l *= f;
                        // the warp rescales its O together (tcgen05.ld / st are warp-wide), rows without need
                        // by 1. The half's previous product is done: S of this tile was issued after it.
                        if (__any_sync(kFull, f != 1.f)) {
#pragma unroll 1
                            for (int ch = 0; ch < 8; ++ch) {
                                uint32_t o[16];
                                tmem_ld16_async(obuf + ch * 16, o);
                                tmem_wait_dep(o);
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tmem_st16(obuf + ch * 16, o);
                            }
                        }
                    }
                    const float mr = m == -INFINITY ? 0.f : -m;
                    const f2 mm = pack2(mr, mr);
                    f2 lsum[4] = {pack2(0.f, 0.f), pack2(0.f, 0.f), pack2(0.f, 0.f), pack2(0.f, 0.f)};
                    uint32_t s0[32], s1[32], s2[32], s3[32], pk[32], pk2[32];
                    tmem_ld32_async(sbuf, s0);
                    tmem_ld32_async(sbuf + 32, s1);
                    tmem_wait_dep(s0);
                    tmem_wait_dep(s1);
                    exp_scores<kF16>(s0, cc, mm, lsum, pk, 0);
                    tmem_ld32_async(sbuf + 64, s2);
                    exp_scores<kF16>(s1, cc, mm, lsum, pk, 16);
                    tmem_ld32_async(sbuf + 96, s3);
                    tmem_wait_dep(s2);
                    tmem_wait_dep(s3);
                    exp_scores<kF16>(s2, cc, mm, lsum, pk2, 0);
                    exp_scores<kF16>(s3, cc, mm, lsum, pk2, 16);
                    float l0, l1;
                    unpack2(add2(add2(lsum[0], lsum[1]), add2(lsum[2], lsum[3])), l0, l1);
                    l0 += l1;
                    raise = live && col.lo < col.hi && (!(l0 < kMostWeight) || (!kF16 && l == 0.f && l0 < kLeastWeight));
                    if (round == 0 && __any_sync(kFull, raise)) continue;
                    l += l0;
                    tmem_st32_u(sbuf, pk);
                    tmem_st32_u(sbuf + 64, pk2);
                    break;
                }
                tmem_wait_st();
            }
            if (x + kStages >= count) c.ml[n & 3][h][r] = make_float2(l == 0.f ? -INFINITY : m, l);
            // (one of the half's warps also waits for V, which is there by now: the issuer then
            // has one wait less)
            if (q == 0 && !(ok = warp_wait(&c.v_full[h], (t / kStages) & 1, c, a))) break;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.p_full[h]);
        }
        t0 += count;
        if (ok) release_piece(n, lane, c);
    }
}

template <bool kF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    return kF16 ? pack_f16(lo, hi) : pack_bf16(lo, hi);
}

// The warp's stage (32 rows x 128 bytes) to the rows' addresses (0: not stored), 4 rows
// of 128 contiguous bytes per instruction. Written a row per thread with the 16-byte
// chunk index XORed with the row's low three bits, so that neither the writes nor the
// reads put two threads of a quarter-warp in one bank group.
__device__ __forceinline__ void store_stage(uint32_t stage, int lane, uint64_t row, uint32_t at) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int rr = i * 4 + (lane >> 3), x = lane & 7;
        const uint64_t to = __shfl_sync(kFull, row, rr);
        const uint4 v = ld_shared_v4(stage + rr * 128 + ((x ^ (rr & 7)) << 4));
        if (to) *reinterpret_cast<uint4 *>(to + at + x * 16) = v;
    }
    __syncwarp();  // (the stage is rewritten next)
}

// The read-out of the CTA's pieces; this thread's row is TMEM lane q * 32 + lane. O is
// handed back to the MMA as soon as it is in registers and the stage: the products
// of the next piece wait for it.
template <bool kF16>
__device__ __forceinline__ void read_out(uint32_t tmem, int q, int lane, uint32_t stage, uint32_t tiles, const Range &range,
                                         const Plan &plan, Ctl &c, const PrefixArgs &a) {
    uint32_t t0 = 0;
    Schedule z;
    const bool scheduler = q == 0;
    if (scheduler) z = schedule_start(a, range, plan, lane, c);
    const int r = q * 32 + lane, tok = prefix::quotient(r, a.s.by_group);
    const uint32_t col = tmem + (static_cast<uint32_t>(q * 32) << 16) + kOCol;
#pragma unroll 1
    for (int n = 0; t0 < tiles; ++n) {
        if (scheduler)
#pragma unroll 1
            while (z.n < n + kRing && schedule_next(z, a, range, lane, c)) {
            }
        const Piece *pp = next_piece(n, c, a);
        if (!pp) return;
        const Piece &p = *pp;
        const int count = p.j1 - p.j0;
        if (p.last) tiles = t0 + count;
        const bool whole = p.part < 0;
        uint64_t row = 0;  // where this thread's row goes, 0: nowhere
        float *lse = nullptr;
        if (tok < p.r.n_tok && p.len[prefix::quotient(p.r.tok0 + tok, a.s.by_n_q) - p.r.b0] >= 0) {
            const int t = p.r.tok0 + tok, h = p.head * a.s.group + r - tok * a.s.group;
            row = whole ? reinterpret_cast<uint64_t>(a.out) + 2 * (p.q * a.out_req + t * a.out_token + h * a.out_head)
                        : reinterpret_cast<uint64_t>(a.part_o + ((2 * blockIdx.x + p.part) * prefix::kRows + r) * kD);
            if (whole && a.lse) lse = a.lse + (static_cast<int64_t>(p.q) * a.s.n_tokens + t) * a.n_heads + h;
        }
        if (!warp_wait(&c.o_ready, n & 1, c, a)) return;
        tc_fence_after();
        const bool both = count > 1;
        const int only = static_cast<int>(t0) & 1;  // the half of a one-tile piece's tile
        const uint32_t at0 = col + (both ? 0 : only * 128), at1 = both ? col + 128 : at0;
        uint32_t o[64], o1[64];  // 64 columns at a time, the first on their way while the weights are computed
        uint32_t(&oa)[32] = *reinterpret_cast<uint32_t(*)[32]>(&o[0]);
        uint32_t(&ob)[32] = *reinterpret_cast<uint32_t(*)[32]>(&o[32]);
        uint32_t(&pa)[32] = *reinterpret_cast<uint32_t(*)[32]>(&o1[0]);
        uint32_t(&pb)[32] = *reinterpret_cast<uint32_t(*)[32]>(&o1[32]);
        const auto load = [&](int from) {
            tmem_ld32_async(at0 + from, oa);
            tmem_ld32_async(at1 + from, pa);
            tmem_ld32_async(at0 + from + 32, ob);
            tmem_ld32_async(at1 + from + 32, pb);
        };
        load(0);
        float2 e = c.ml[n & 3][both ? 0 : only][r];
        float2 f = both ? c.ml[n & 3][1][r] : make_float2(-INFINITY, 0.f);
        const float m = fmaxf(e.x, f.x), mr = m == -INFINITY ? 0.f : m;
        float w0 = e.y == 0.f ? 0.f : ex2(e.x - mr), w1 = f.y == 0.f ? 0.f : ex2(f.x - mr);
        const float l = w0 * e.y + w1 * f.y;  // (NaN stays)
        if (whole) {
            const float inv = l == 0.f ? 0.f : __fdividef(1.f, l);
            w0 *= inv;
            w1 *= inv;
        }
        // (what has no weight may hold anything, NaN too: its bits are cleared)
        const uint32_t keep0 = w0 == 0.f ? 0u : ~0u, keep1 = w1 == 0.f ? 0u : ~0u;
        const bool zeros = __any_sync(kFull, (keep0 & keep1) == 0);
        const f2 ww0 = pack2(w0, w0), ww1 = pack2(w1, w1);
#pragma unroll 1
        for (int it = 0; it < 3; ++it) {  // what was staged leaves a turn later
            if (it < 2) {
                tmem_wait_dep(oa);
                tmem_wait_dep(pa);
                tmem_wait_dep(ob);
                tmem_wait_dep(pb);
            }
            if (it == 1) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&c.o_free);  // O may take the next piece
            }
            if (it > 0 && whole) store_stage(stage, lane, row, (it - 1) * 128);
            if (it == 2) break;
            if (zeros) {
#pragma unroll
                for (int i = 0; i < 64; ++i) {
                    o[i] &= keep0;
                    o1[i] &= keep1;
                }
            }
#pragma unroll
            for (int i = 0; i < 64; i += 2) {
                const f2 x = pack2(__uint_as_float(o[i]), __uint_as_float(o[i + 1]));
                const f2 y = pack2(__uint_as_float(o1[i]), __uint_as_float(o1[i + 1]));
                float lo, hi;
                unpack2(fma2(y, ww1, mul2(x, ww0)), lo, hi);
                if (whole) {
                    o[i / 2] = pack16<kF16>(lo, hi);
                } else {
                    o[i] = __float_as_uint(lo);
                    o[i + 1] = __float_as_uint(hi);
                }
            }
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {  // (32 columns of fp32 fill the stage, 64 of 16 bits)
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    st_shared_v4(stage + lane * 128 + ((u ^ (lane & 7)) << 4),
                                 make_uint4(o[4 * u], o[4 * u + 1], o[4 * u + 2], o[4 * u + 3]));
                if (whole) break;
                store_stage(stage, lane, row, it * 256 + half * 128);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = o[32 + i];
            }
            if (it == 0) load(64);
        }
        if (lse) *lse = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
        if (!whole) a.part_ml[(2 * blockIdx.x + p.part) * prefix::kRows + r] = make_float2(m, l);
        t0 += count;
        release_piece(n, lane, c);
    }
}

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 1)
    prefix_attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                            const __grid_constant__ CUtensorMap tm_v, const PrefixArgs a) {
    extern __shared__ uint8_t dyn_smem[];
    __shared__ Ctl c;
    const int warp = __shfl_sync(kFull, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    uint8_t *base = dyn_smem + ((1024u - (saddr(dyn_smem) & 1023u)) & 1023u);
    uint8_t *sq = base;                          // Q buffers
    uint8_t *sk = sq + kQBufs * kTileBytes;      // K stages
    uint8_t *sv = sk + kStages * kTileBytes;     // V stages
    uint8_t *so = sv + kStages * kTileBytes;     // output stages of the read-out warps
    if (threadIdx.x == 0) {
        for (int b = 0; b < kQBufs; ++b) mbar_init(&c.q_full[b], 1);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&c.k_full[s], 1);
            mbar_init(&c.v_full[s], 1);
            mbar_init(&c.v_empty[s], 1);
            mbar_init(&c.v_raw[s], 1);
            mbar_init(&c.s_full[s], 1);
            mbar_init(&c.p_full[s], 4);  // a half's four warps
        }
        for (int s = 0; s < kRing; ++s) {
            mbar_init(&c.ring_full[s], 1);
            mbar_init(&c.ring_empty[s], kConsumers);
        }
        mbar_init(&c.o_ready, 1);
        mbar_init(&c.o_free, 4);
        mbar_init(&c.mma_done, 1);
        c.abort_flag = 0;
        for (const CUtensorMap *m : {&tm_q, &tm_k, &tm_v})
            asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        tmem_alloc(&c.tmem_base, kTmemCols);
        tmem_relinquish();
    }
    pdl_wait();
    pdl_launch_next();
    if (threadIdx.x == 0 && !a.by_tile) a.cut[blockIdx.x].parts = 0;
    const Plan plan{reinterpret_cast<int64_t *>(sk), reinterpret_cast<Tiles *>(sq)};
    const Range range = find_range(a, c, plan);
    // (the copies that follow are ordered after the plan's writes)
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = c.tmem_base;
    const uint32_t tiles = range.at < range.end ? kNoEnd : 0;  // (each role learns the end from its last piece)

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCtlRegs));
        if (warp == 0 || warp == 2)
            produce(warp == 0, warp == 0 ? &tm_k : &tm_v, &tm_q, warp == 0 ? sk : sv, sq, tiles, lane, c, a);
        else if (warp == 1)
            issue_products<kF16>(sq, sk, sv, tmem, tiles, lane, c, a);
        else
            clean(sv, tiles, lane, c, a);
    } else if (warp < 12) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
        softmax<kF16>(tmem, warp & 3, lane, (warp >> 2) - 1, tiles, c, a);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kOutRegs));
        if (tiles) read_out<kF16>(tmem, warp & 3, lane, saddr(so + (warp - 12) * kStageBytes), tiles, range, plan, c, a);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && c.abort_flag) flag_error(a.err, RPS_DEVERR_TIMEOUT);
    if (warp == 1) tmem_dealloc(tmem, kTmemCols);
}

// ---------------------------------------------------------------- joining the parts of cut row tiles
// Half a warp takes a row's parts first, first + step, ..., a lane eight of its columns.
struct Joined {
    float m, l;
    float4 o[2];
};
__device__ __forceinline__ void weigh(float4 &x, float f, const float4 &y, float g) {
    x.x = x.x * f + y.x * g;
    x.y = x.y * f + y.y * g;
    x.z = x.z * f + y.z * g;
    x.w = x.w * f + y.w * g;
}
__device__ __forceinline__ void join(Joined &x, float m, float l, const float4 (&o)[2]) {
    const float mm = fmaxf(x.m, m), mr = mm == -INFINITY ? 0.f : mm;
    const float f = ex2(x.m - mr), g = ex2(m - mr);
    x.m = mm;
    x.l = x.l * f + l * g;
    weigh(x.o[0], f, o[0], g);
    weigh(x.o[1], f, o[1], g);
}

constexpr int kJoinThreads = 128, kJoinHalves = kJoinThreads / 16;
constexpr int kAhead = 4;  // parts in flight

// Block (cut, group of rows): `split` half warps share a row. Most cuts have two or
// three parts; with few row tiles there are many, and the row's parts are split.
template <bool kF16>
__global__ void __launch_bounds__(kJoinThreads) prefix_combine_kernel(const PrefixArgs a, int split) {
    __shared__ Joined others[kJoinHalves][16];
    const int half = threadIdx.x >> 4, lane = threadIdx.x & 15;
    pdl_wait();
    pdl_launch_next();
    Cut cut = a.cut[blockIdx.x];
    if (a.by_tile) {  // (the entry of a row tile without a sequence is not written: its lengths say so)
        const int qh = prefix::quotient(blockIdx.x, a.s.by_row_tiles);
        cut.rt = blockIdx.x - qh * a.s.row_tiles;
        cut.q = qh / a.s.heads;
        cut.head = qh - cut.q * a.s.heads;
    } else if (cut.parts == 0) {
        return;
    }
    const RowTile r = prefix::row_tile(a.s, cut.rt);
    const int row = blockIdx.y * (kJoinHalves / split) + half / split, which = half % split;
    const int t = prefix::quotient(row, a.s.by_group), tok = r.tok0 + t;
    // (a call that gave up may not have written its entries: the parts are kept inside the workspace)
    const bool there = t < r.n_tok && a.len[cut.q * a.s.n_branch + prefix::quotient(tok, a.s.by_n_q)] >= 0 &&
                       cut.parts > 0 && cut.cta >= 0 && cut.cta < kMaxCtas && cut.parts <= kMaxCtas - cut.cta;
    Joined x{-INFINITY, 0.f, {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)}};
    if (there) {
#pragma unroll 1
        for (int p = which; p < cut.parts; p += split * kAhead) {
            float2 ml[kAhead];
            float4 o[kAhead][2];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int pp = min(p + u * split, cut.parts - 1);
                // the first part of a row tile ends its CTA's range, the others begin theirs
                const int64_t at = static_cast<int64_t>(2 * (cut.cta + pp) + (pp == 0 ? 1 : 0)) * prefix::kRows + row;
                ml[u] = a.part_ml[at];
                o[u][0] = *reinterpret_cast<const float4 *>(a.part_o + at * kD + lane * 8);
                o[u][1] = *reinterpret_cast<const float4 *>(a.part_o + at * kD + lane * 8 + 4);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (p + u * split < cut.parts) join(x, ml[u].x, ml[u].y, o[u]);
        }
    }
    if (split > 1) {
        others[half][lane] = x;
        __syncthreads();
        if (which) return;
#pragma unroll 1
        for (int w = 1; w < split; ++w) {
            const Joined y = others[half + w][lane];
            join(x, y.m, y.l, y.o);
        }
    }
    if (!there) return;
    const int h = cut.head * a.s.group + row - t * a.s.group;
    const float inv = x.l == 0.f ? 0.f : 1.f / x.l;
    const uint4 v = make_uint4(pack16<kF16>(x.o[0].x * inv, x.o[0].y * inv), pack16<kF16>(x.o[0].z * inv, x.o[0].w * inv),
                               pack16<kF16>(x.o[1].x * inv, x.o[1].y * inv), pack16<kF16>(x.o[1].z * inv, x.o[1].w * inv));
    *reinterpret_cast<uint4 *>(static_cast<char *>(a.out) +
                               (cut.q * a.out_req + tok * a.out_token + h * a.out_head + lane * 8) * 2) = v;
    if (a.lse && lane == 0)
        a.lse[(static_cast<int64_t>(cut.q) * a.s.n_tokens + tok) * a.n_heads + h] =
            x.l == 0.f ? -INFINITY : (x.m + log2f(x.l)) * kLn2;
}

// ---------------------------------------------------------------- host
std::mutex g_prefix_mutex;
PFN_cuTensorMapEncodeTiled_v12000 g_prefix_encode = nullptr;
bool g_prefix_ready[64] = {};
int g_prefix_sms[64] = {};

rps_status setup(int *sms) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RPS_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g_prefix_mutex);
    if (!g_prefix_encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) !=
                cudaSuccess ||
            q != cudaDriverEntryPointSuccess || !fn)
            return RPS_ERR_CUDA;
        g_prefix_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }
    if (!g_prefix_ready[dev]) {
        if (cudaDeviceGetAttribute(&g_prefix_sms[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
            return RPS_ERR_CUDA;
        for (auto k : {prefix_attention_kernel<false>, prefix_attention_kernel<true>})
            if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess)
                return RPS_ERR_CUDA;
        g_prefix_ready[dev] = true;
    }
    *sms = std::min(g_prefix_sms[dev], kMaxCtas);
    return RPS_OK;
}

// A map of 16-bit elements: extents, strides (in elements) and boxes from the inner dimension
// (64-wide boxes of kD contiguous elements, or 64) outwards.
template <int n>
rps_status make_map(CUtensorMap *m, const void *base, bool f16, int64_t inner, const int64_t (&ext)[n],
                    const int64_t (&stride)[n], const uint32_t (&box)[n]) {
    cuuint64_t dims[n + 1] = {static_cast<cuuint64_t>(inner)}, bytes[n];
    cuuint32_t boxes[n + 1] = {64}, es[n + 1] = {1};
    for (int i = 0; i < n; ++i) {
        dims[i + 1] = static_cast<cuuint64_t>(ext[i]);
        // (the stride of a dimension of one is not used, but has to be a valid one)
        bytes[i] = static_cast<cuuint64_t>(ext[i] > 1 ? stride[i] : kD) * 2;
        boxes[i + 1] = box[i];
        es[i + 1] = 1;
    }
    const CUresult r = g_prefix_encode(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, n + 1,
                                       const_cast<void *>(base), dims, bytes, boxes, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? RPS_OK : RPS_ERR_CUDA;
}

// The maps of K and V: a copy brings whole groups of 8 tokens, both halves of their columns.
// Where the pages' stride is a multiple of eight tokens', one dimension goes through the groups
// of all pages, and a copy takes a slot; else a copy is a group of one page.
rps_status map_pages(CUtensorMap *tk, CUtensorMap *tv, const rps_kv_cache *kv, int64_t layer_at, bool f16, PrefixArgs &a) {
    const int64_t groups = kv->page_size / 8, token = kv->token_stride, group = 8 * token;
    const int64_t per_page = kv->n_pages > 1 ? kv->page_stride / group : groups;
    const int64_t all = (kv->n_pages - 1) * per_page + groups;
    const void *const base[2] = {static_cast<char *>(kv->k) + layer_at, static_cast<char *>(kv->v) + layer_at};
    CUtensorMap *const to[2] = {tk, tv};
    a.by_groups = (kv->n_pages == 1 || kv->page_stride % group == 0) && all <= INT32_MAX;
    a.copy_log = a.by_groups ? a.s.slot_log : 3;
    a.page_groups = a.by_groups ? static_cast<int32_t>(per_page) : 0;
    a.no_page = a.by_groups ? static_cast<int32_t>(all) : kv->n_pages;
    for (int i = 0; i < 2; ++i) {
        rps_status st;
        if (a.by_groups) {
            const int64_t ext[4] = {8, 2, all, kv->n_heads}, stride[4] = {token, 64, group, kv->head_stride};
            const uint32_t box[4] = {8, 2, static_cast<uint32_t>(a.s.slot / 8), 1};
            st = make_map(to[i], base[i], f16, 64, ext, stride, box);
        } else {
            const int64_t ext[4] = {kv->page_size, 2, kv->n_heads, kv->n_pages};
            const int64_t stride[4] = {token, 64, kv->head_stride, kv->page_stride};
            const uint32_t box[4] = {8, 2, 1, 1};
            st = make_map(to[i], base[i], f16, 64, ext, stride, box);
        }
        if (st != RPS_OK) return st;
    }
    return RPS_OK;
}

// Shape of a call, with the limits that keep its counts in 32 bits.
rps_status check_shape(const rps_kv_cache *kv, int32_t n_q, int32_t n_heads, int32_t causal, Shape *s) {
    const rps_status st = check_kv_cache(kv);
    if (st != RPS_OK) return st;
    if (n_q < 1 || n_heads < 1 || n_heads % kv->n_heads) return RPS_ERR_INVALID_ARG;
    if (n_heads / kv->n_heads > RPS_KV_MAX_GROUP) return RPS_ERR_UNSUPPORTED;
    const int64_t tokens = static_cast<int64_t>(kv->n_branch) * n_q;
    if (tokens > INT32_MAX / 256 || static_cast<int64_t>(kv->n_req) * tokens > INT32_MAX / 256) return RPS_ERR_UNSUPPORTED;
    if (kv->n_req > kMaxReqs) return RPS_ERR_UNSUPPORTED;
    // slots of the sequences of one row tile
    const int64_t slots = static_cast<int64_t>(kv->max_pages) * std::max(1, kv->page_size / prefix::kRows);
    if (std::min<int64_t>(kv->n_branch, kMaxSeqs) * slots > INT32_MAX / 256) return RPS_ERR_UNSUPPORTED;
    *s = prefix::make_shape(kv->n_req, kv->n_branch, n_q, kv->n_heads, n_heads / kv->n_heads, kv->page_size, kv->n_pages,
                            kv->max_pages, causal);
    return RPS_OK;
}

size_t part_bytes(size_t *ml_at, size_t *o_at) {
    *ml_at = (sizeof(Cut) * kMaxCtas + 255) / 256 * 256;
    *o_at = *ml_at + sizeof(float2) * 2 * kMaxCtas * prefix::kRows;
    return *o_at + sizeof(float) * 2 * kMaxCtas * prefix::kRows * kD;
}

}  // namespace
}  // namespace rps

using namespace rps;

extern "C" size_t rps_prefix_attention_workspace_bytes(const rps_kv_cache *kv, int32_t n_q, int32_t n_heads) {
    Shape s;
    if (check_shape(kv, n_q, n_heads, 0, &s) != RPS_OK) return 0;
    size_t ml, o;
    return part_bytes(&ml, &o);
}

extern "C" rps_status rps_prefix_attention_fwd(const rps_prefix_attention *p, const rps_kv_cache *kv, void *d_ws,
                                               size_t ws_bytes, rps_stream_t stream) {
    if (!p || !p->q || !p->out) return RPS_ERR_INVALID_ARG;
    PrefixArgs a;
    std::memset(&a, 0, sizeof a);
    rps_status st = check_shape(kv, p->n_q, p->n_heads, p->causal != 0, &a.s);
    if (st != RPS_OK) return st;
    if (p->layer < 0 || p->layer >= kv->n_layers) return RPS_ERR_INVALID_ARG;
    if (!(p->scale > 0.f) || !std::isfinite(p->scale)) return RPS_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p->q) % 16 || reinterpret_cast<uintptr_t>(p->out) % 16) return RPS_ERR_INVALID_ARG;
    const int64_t ext[3] = {p->n_heads, a.s.n_tokens, kv->n_req};
    const int64_t qs[3] = {p->q_head_stride, p->q_token_stride, p->q_req_stride};
    const int64_t os[3] = {p->out_head_stride, p->out_token_stride, p->out_req_stride};
    for (int i = 0; i < 3; ++i)
        if (ext[i] > 1 && (qs[i] <= 0 || os[i] <= 0 || qs[i] % 8 || os[i] % 8)) return RPS_ERR_INVALID_ARG;
    size_t ml_at, o_at;
    if (!d_ws || reinterpret_cast<uintptr_t>(d_ws) % 16 || ws_bytes < part_bytes(&ml_at, &o_at))
        return RPS_ERR_INVALID_ARG;
    int sms = 0;
    if ((st = setup(&sms)) != RPS_OK) return st;
    if (!(a.err = device_error_word())) return RPS_ERR_CUDA;

    const bool f16 = kv->dtype == RPS_F16;
    const int64_t kv_at = kv->n_layers > 1 ? p->layer * kv->layer_stride * 2 : 0;
    const uint32_t qbox[3] = {static_cast<uint32_t>(a.s.group), static_cast<uint32_t>(a.s.tokens), 1};
    CUtensorMap tq, tk, tv;
    if ((st = make_map(&tq, p->q, f16, kD, ext, qs, qbox)) != RPS_OK) return st;
    if ((st = map_pages(&tk, &tv, kv, kv_at, f16, a)) != RPS_OK) return st;
    a.table = kv->table;
    a.len = kv->len;
    a.shared_len = p->shared_len;
    a.n_heads = p->n_heads;
    a.out = p->out;
    a.out_req = kv->n_req > 1 ? os[2] : 0;
    a.out_token = a.s.n_tokens > 1 ? os[1] : 0;
    a.out_head = p->n_heads > 1 ? os[0] : 0;
    a.lse = p->lse;
    a.c = p->scale * kLog2e;
    char *ws = static_cast<char *>(d_ws);
    a.cut = reinterpret_cast<Cut *>(ws);
    a.part_ml = reinterpret_cast<float2 *>(ws + ml_at);
    a.part_o = reinterpret_cast<float *>(ws + o_at);
    a.tries = static_cast<uint32_t>(std::min<uint64_t>((ring_wait_limit_ns() + 999) / 1000, 1u << 30));

    // CTAs: as many as there can be key tiles
    const int64_t slots = static_cast<int64_t>(a.s.max_pages) * a.s.sub;
    const int64_t tiles = 2 + (std::min<int64_t>(a.s.n_branch, kMaxSeqs) + 1) * slots / a.s.spt;
    const int64_t row_tiles = static_cast<int64_t>(a.s.n_req) * a.s.heads * a.s.row_tiles;
    const int grid = static_cast<int>(std::min<int64_t>(row_tiles * tiles, sms));
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const prefix::CutList list = prefix::cut_list(row_tiles, grid);
    a.by_tile = list.by_tile;
    if (launch_pdl(f16 ? prefix_attention_kernel<true> : prefix_attention_kernel<false>, dim3(grid), dim3(kThreads),
                   kSmemBytes, s, tq, tk, tv, a) != cudaSuccess)
        return RPS_ERR_CUDA;
    // a cut row tile has about grid / row_tiles parts: half warps of at most four each (64 sequences
    // of one prompt, 16 row tiles: 2.4 us faster than with one half warp a row)
    int split = 1;
    while (split < kJoinHalves && row_tiles * kAhead * split < grid) split *= 2;
    const dim3 cuts(static_cast<unsigned>(list.blocks), prefix::kRows / (kJoinHalves / split));
    return launch_pdl(f16 ? prefix_combine_kernel<true> : prefix_combine_kernel<false>, cuts, dim3(kJoinThreads), 0, s, a,
                      split) == cudaSuccess
               ? RPS_OK
               : RPS_ERR_CUDA;
}
