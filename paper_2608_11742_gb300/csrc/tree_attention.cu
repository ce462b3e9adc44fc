// tree_attention.cu -- attention of each sequence's drafted tokens over the paged K/V
// cache, with a mask of their own over each other (rps_tree_attention_fwd).
//
// For query i, out = sum_j softmax_j(scale q . k_j) v_j over the context and the drafted
// tokens whose bits its mask has. The softmax over two sets of keys is joined from the
// sets' maxima m, sums l and weighted sums o: with m = max(m1, m2) both sides are weighted
// by 2^(m_x - m) and added. So the query rows that share a cache head (drafted tokens times
// query heads) are stacked as the 128 rows of one matrix product with the keys, and the
// key tiles of all (sequence, head)s are dealt to the CTAs in equal parts (tree_split.h),
// whose partial (m, l, o) a second launch joins.
//
// One persistent CTA per SM takes pieces (unit, key tiles [j0, j1)). A piece is a list of
// items, a row tile with a key tile each, that alternate between two halves of the softmax
// with an S / P buffer and an accumulator of their own. A unit of two row tiles gives each
// key tile to both, a half each: the keys are read once for 256 rows. A unit of one gives
// even key tiles to one half and odd ones to the other, which are added up at the end.
//   warp 0      TMA producer of K, one box per slot of pages, addresses through the page
//               table, and of Q (a box of tokens x heads of the group);
//   warp 2      TMA producer of V. V lies token by token in the cache, so it is the MN-major
//               operand of the second product: no transposed copy of the values is kept;
//   warp 1      MMA issuer, one thread: S = Q K^T into the half's TMEM buffer, O += P V with
//               P from TMEM, in the order PV(x), S(x + 2), PV(x + 1), ...;
//   warps 4-7   softmax of even items, 8-11 of odd ones: thread = row. One pass with a
//               standing base-2 reference, which is changed only where a tile's sum is far
//               out of range. P is rounded to the cache's type (the product takes no other);
//               its sum is taken before the rounding, in fp32. The output's error is 1.4 times that of
//               its own rounding so (bf16 0.0023 instead of 0.0017, root mean square); P in two parts
//               brings it back, at 101 us instead of 98 for 64 single tokens and 208 instead of 172 for
//               64 x 1, 32 / 32 heads, context 1000. Before the last key tile's P is
//               handed on, V's rows past the sequence's end are cleared (they may hold
//               anything, and 0 * NaN would reach the sums). At a piece's end the same warps
//               read the accumulators out.
//
// What bounds it, at the figures measured (times of both launches, warm, from a graph):
//   64 sequences x 1 token, 28 / 4 heads, contexts 200 to 8000: 90 us, 5.97 TB/s, 0.88 of a copy's
//     bandwidth. 64 x 1, 32 / 32 heads, context 1000: 167 us, 0.93.
//   2 sequences x 64 tokens, 32 / 8 heads, contexts 24000 to 32700, fp16: 60 us, 3.9 TB/s; 64 x 1 to 32
//     tokens, 32 / 4 heads, contexts 500 to 4000: 75 us, 4.2 TB/s. A pair's key tile takes 1.6 to 1.85 us,
//     1.47 at HBM's rate: its products read 192 KB of shared memory and the copies write 64 (2048 cycles),
//     and a half's next scores wait for its softmax (1580 cycles), P V and their own product. Slower: S and P
//     in halves of 64 keys (65 -> 71), two warps to 32 rows in the softmax (60 -> 63).
//   Start and end: the range is known 1.9 us after the launch before has ended, the first scores are there
//     2.7 to 4.3 later, the last CTA ends 4 to 6 us after the median one, the joining launch takes 4 to 8.
//   200 sequences x 4 tokens, 32 / 8 heads, contexts 20 to 300: 57 us, 10 units a CTA of two key tiles each; 77 with
//     a third more code in the roles, which have to fit the instruction cache together.
// Every wait is bounded; a role whose wait runs out flags RPS_DEVERR_TIMEOUT and raises the
// CTA's abort flag, copies and MMAs in flight are drained and TMEM is freed before the CTA
// exits.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "kv_maps.cuh"
#include "rps_internal.cuh"
#include "tc_device.cuh"
#include "tree_split.h"
#include "umma_desc.h"

namespace rps {
namespace {

using tree::kMaxCtas;
using tree::Piece;
using tree::Seq;
using tree::Shape;
using tree::Walk;

constexpr int kD = kHeadDim;
constexpr int kAtom = 64 * 128 * 2;    // one 128-row x 64-column swizzle atom of 16-bit elements: 16 KB
constexpr int kTileBytes = 2 * kAtom;  // a Q, K or V tile: Q's two atoms along d
// A K or V tile goes in groups of 8 tokens: their columns 0..63, then 64..127 (1024 bytes each).
constexpr int kChunk = 1024, kGroup = 2 * kChunk;
constexpr int kStages = 2;  // of K and of V
constexpr int kQBufs = 2;   // two pieces' row tile, or the two row tiles of one
constexpr int kSmemBytes = kQBufs * kTileBytes + 2 * kStages * kTileBytes + 1024;
constexpr int kThreads = 384;
constexpr uint32_t kTmemCols = 512;  // S buffers at columns 0 and 128, O at 256 and 384
constexpr uint32_t kOCol = 256;
constexpr int kWholeTiles = 4;       // key tiles of units that are never cut
constexpr int kMlSlots = 3;
constexpr int kStagedSeqs = 1024;    // sequences whose lengths are kept in shared memory
constexpr float kLn2 = 0.6931471805599453f;
// bounds of a tile's sum of P in a row (in units of its reference): P in fp16 stays finite
constexpr float kMostWeight = 32768.f, kLeastWeight = 1.f / 32768.f;

// A unit that is cut: the CTA that takes its first key tile writes where its parts are.
struct __align__(16) Cut {
    int32_t parts;                // 0: none; else on this CTA and the next ones
    int32_t cta, s, h, p, count;  // count: queries of the sequence
    int32_t pad[2];
};

struct TreeArgs {
    Shape s;
    const int32_t *table, *len, *count;
    const uint32_t *mask;
    int32_t words;    // of a query's mask
    int32_t n_heads;  // query heads
    void *out;
    int64_t out_seq, out_token, out_head;
    float *lse;
    float c;  // scale * log2(e)
    PageCopies copies;
    int32_t paired;   // units may have two row tiles
    int32_t few;      // no more units than CTAs, and a thread for each sequence
    int32_t whole;    // and none is cut: a CTA takes one
    int32_t sectors;  // output rows begin on 32-byte bounds
    Cut *cut;         // [grid]
    float2 *part_ml;  // [2 * grid][2][128]: maximum and sum of each row of a partial result
    float *part_o;    // [2 * grid][2][128][128]
    uint32_t *err;
    uint32_t tries;  // of a wait
};

// A piece, and the items before it.
struct Noted {
    Piece p;
    uint32_t x0;
};

struct Ctl {
    uint64_t q_full[kQBufs], q_empty[kQBufs], k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
    uint64_t s_full[2], p_full[2], o_ready, o_free, mma_done;
    // a half's reference and sum of a row at the end of piece n, in slot n % 3: written before the half's last
    // P of the piece is handed on, read once O is ready, and written again for piece n + 3 by warps that have
    // seen O of piece n + 1 ready, whose products wait for the read-out of n
    float2 ml[kMlSlots][2][tree::kRows];
    Noted noted[8];  // of each warp of the softmax: the piece that it has to read out
    int4 copy_at[2][32];  // a producer's copies: their coordinates, of two tiles
    uint32_t bad[4];      // copies of key tile t whose page id is outside the cache (t % 4)
    Seq seq[kStagedSeqs];  // as they are used
    int64_t scan[kThreads / 32];
    Walk walk;
    int64_t range_end;
    tree::Ranges ranges;
    int longest;
    uint32_t tmem_base;
    int abort_flag;
};

__device__ __forceinline__ Seq seq_of(const TreeArgs &a, int s) {
    return tree::used_seq(a.s, a.len[s], a.count ? a.count[s] : a.s.n_q);
}

// Exclusive prefix sum over the block's threads; *total: the block's sum.
__device__ __forceinline__ int64_t scan_block(int64_t v, int64_t *sums, int64_t *total) {
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

// The CTA's range of the places of all units, or its one unit, as c.walk (left 0: nothing to do).
__device__ __forceinline__ void find_range(const TreeArgs &a, Ctl &c) {
    const int n_seq = a.s.n_seq;
    if (threadIdx.x == 0) {
        c.longest = 0;
        c.walk = Walk{0, 0, 0, 0, 0};
    }
    // the places of the sequences
    int64_t places = 0, work = 0, before = 0, total;
    Seq q{-1, 0};
    int longest = 0;
    const auto look = [&](int e) {
        q = e < n_seq ? seq_of(a, e) : Seq{-1, 0};
        if (e < n_seq && n_seq <= kStagedSeqs) c.seq[e] = q;
        places = tree::places_of(a.s, q, &longest);
    };
    // The CTA's unit by its number. (A thread has its sequence.)
    const auto take_unit = [&](int me) {
        const int pairs = tree::pairs_of(a.s, q), units = pairs * a.s.heads;
        const int first = static_cast<int>(scan_block(units, c.scan, &total));
        if (me >= first && me < first + units) {
            const int u = me - first, h = u / pairs, p = u - h * pairs;
            c.walk = Walk{static_cast<int>(threadIdx.x), h, p, 0, tree::cost_of(a.s, q, p)};
        }
    };
    const int grid = gridDim.x, me = blockIdx.x;
    if (a.whole) {
        look(threadIdx.x);
        return take_unit(me);
    }
#pragma unroll 1
    for (int base = 0; base < n_seq; base += kThreads) {
        look(base + threadIdx.x);
        before = scan_block(places, c.scan, &total);
        work += total;
    }
    if (a.few) {
        const int most = __reduce_max_sync(kFull, longest);
        if ((threadIdx.x & 31) == 0 && most) atomicMax(&c.longest, most);
        __syncthreads();
        if (c.longest <= tree::divide(work, grid) + tree::kCutCost) return take_unit(me);
    }
    if (work == 0) return;
    const int n = work < static_cast<int64_t>(grid) * tree::kPairCost ? max(1, static_cast<int>(work) / tree::kPairCost) : grid;
    if (me >= n) return;
    const tree::Ranges r = tree::make_ranges(work, n);
    const int64_t at = tree::range_start(r, me), end = tree::range_start(r, me + 1);
    if (threadIdx.x == 0) {
        c.ranges = r;
        c.range_end = end;
    }
    int64_t carry = 0;
#pragma unroll 1
    for (int base = 0; base < n_seq; base += kThreads) {
        if (n_seq > kThreads) {
            look(base + threadIdx.x);
            before = carry + scan_block(places, c.scan, &total);
            carry += total;
        }
        if (before <= at && at < before + places)
            c.walk = tree::begin_walk(a.s, base + threadIdx.x, q, at - before, end - at);
    }
}

// ---------------------------------------------------------------- roles
__device__ __forceinline__ bool next(const TreeArgs &a, const Ctl &c, Walk &w, Piece &x) {
    return tree::next_piece(a.s, w, x, [&](int s) { return a.s.n_seq <= kStagedSeqs ? c.seq[s] : seq_of(a, s); });
}

// The producers of K (with Q) and of V, in one body: two warps run it.
__device__ __forceinline__ void produce(bool is_k, const CUtensorMap *tm, const CUtensorMap *tm_q, uint8_t *stages,
                                        uint8_t *sq, int lane, Ctl &c, const TreeArgs &a) {
    Walk w = c.walk;
    Piece p{}, following{};
    uint32_t t = 0;
    int n_q = 0;
    bool ok = true;
    uint64_t *full = is_k ? c.k_full : c.v_full, *empty = is_k ? c.k_empty : c.v_empty;
    const int copies = tree::kRows >> a.copies.copy_log;  // of a tile, 16 at most
    const int half = lane >> 4;
    // the page of copy lane % 16 of key tile j of a piece (-1: not a token of the sequence; n_pages: an id outside the cache)
    const auto page_of = [&](const Piece &x, int j, int &token) -> int {
        token = j * tree::kRows + ((lane & 15) << a.copies.copy_log);
        if ((lane & 15) >= copies || j >= x.j1 || token >= x.q.len) return -1;
        return min(static_cast<uint32_t>(a.table[static_cast<int64_t>(x.s) * a.s.max_pages + (token >> a.s.page_log)]),
                   static_cast<uint32_t>(a.s.n_pages));
    };
    // A piece ahead: its first pages' ids are on their way while the piece before is copied, and its
    // queries in L2 (a change of units took 4.5 us, of which the lookups were 2).
    bool some = true;
    int token = 0, id = -1;
#pragma unroll 1
    for (int n = -1; ok && some; ++n) {
        p = following;
        some = next(a, c, w, following);
        int first_token = 0;
        const int first_id = some ? page_of(following, following.j0 + half, first_token) : -1;
        if (n < 0) {  // (p is none yet)
            id = first_id;
            token = first_token;
            continue;
        }
        if (is_k && some && elect_one())
#pragma unroll 1
            for (int r = 0; r < 2 * following.rt; ++r)
                tma_prefetch_4d(tm_q, r & 1 ? 64 : 0, following.h * a.s.group, (2 * following.p + (r >> 1)) * a.s.tokens, following.s);
#pragma unroll 1
        for (int j = p.j0; ok && j < p.j1; j += 2) {
            const int two = min(2, p.j1 - j);
            const bool there = id >= 0, bad_page = id == a.s.n_pages;
            const int in_page = token & ((1 << a.s.page_log) - 1);
            const bool none = !there || bad_page;  // (a coordinate whose copy is all zeros)
            c.copy_at[is_k][lane] = a.copies.by_groups
                                        ? make_int4(0, none ? a.copies.no_page : id * a.copies.page_groups + (in_page >> 3), p.h, 0)
                                        : make_int4(in_page, p.h, none ? a.copies.no_page : id, 0);
            const uint32_t bad = __ballot_sync(kFull, there && bad_page);
            if (bad && is_k && lane == 0) flag_error(a.err, RPS_DEVERR_PAGE);
            __syncwarp();
            if (j + 2 < p.j1) {
                id = page_of(p, j + 2 + half, token);  // (on its way while these copies wait for their stages)
            } else {
                id = first_id;
                token = first_token;
            }
            int done = 0;
            if (elect_one()) {
#pragma unroll 1
                for (; done < two; ++done) {
                    const uint32_t x = t + done;
                    const int s = x % kStages;
                    if (x >= kStages && !lane_wait(&empty[s], (x / kStages - 1) & 1, c, a)) break;
                    // (before the arrival, which hands it on to the softmax of tile x; that of tile x - 4 has read its own)
                    if (is_k) c.bad[x % 4] = bad >> done * 16 & 0xffffu;
                    mbar_expect_tx(&full[s], kTileBytes);
                    uint8_t *dst = stages + s * kTileBytes;
                    const int4 *from = &c.copy_at[is_k][done * 16];
                    int4 at = from[0];
#pragma unroll 1
                    for (int i = 1; i <= copies; ++i, dst += kGroup / 8 << a.copies.copy_log) {
                        const int4 after = from[i & 15];
                        tma_load_5d(dst, tm, 0, at.x, 0, at.y, at.z, &full[s]);
                        at = after;
                    }
                    if (is_k && j + done == p.j0) {
                        // Q, once the scores of the buffer's last piece are computed
                        const int b = a.paired ? 0 : n & 1, uses = a.paired ? n : n >> 1;
                        if (uses > 0 && !lane_wait(&c.q_empty[b], (uses - 1) & 1, c, a)) {
                            ++done;
                            ok = false;
                            break;
                        }
                        mbar_expect_tx(&c.q_full[b], 2u * p.rt * a.s.group * a.s.tokens * 128);
#pragma unroll 1
                        for (int r = 0; r < p.rt; ++r) {
                            uint8_t *to = sq + (b + r) * kTileBytes;
                            const int tok0 = (2 * p.p + r) * a.s.tokens;
                            tma_load_4d(to, tm_q, 0, p.h * a.s.group, tok0, p.s, &c.q_full[b]);
                            tma_load_4d(to + kAtom, tm_q, 64, p.h * a.s.group, tok0, p.s, &c.q_full[b]);
                        }
                        ++n_q;
                    }
                }
            }
            done = __reduce_max_sync(kFull, done);
            n_q = __reduce_max_sync(kFull, n_q);
            ok = __all_sync(kFull, ok) && done == two;
            t += done;
        }
    }
    // every copy issued lands before the CTA leaves
    if (lane == 0) {
#pragma unroll 1
        for (uint32_t x = t > kStages ? t - kStages : 0; x < t; ++x) drain(&full[x % kStages], (x / kStages) & 1);
        if (a.paired) {
            if (n_q) drain(&c.q_full[0], (n_q - 1) & 1);
        } else {
#pragma unroll 1
            for (int x = n_q > kQBufs ? n_q - kQBufs : 0; x < n_q; ++x) drain(&c.q_full[x & 1], (x >> 1) & 1);
        }
    }
    __syncwarp();
}

// The MMA issuer, one thread. The tensor pipe runs the products in order, so S of item x + 2 may
// overwrite the P that the product of item x reads without a wait.
template <bool kF16>
__device__ __forceinline__ void issue_products(uint8_t *sq, uint8_t *sk, uint8_t *sv, uint32_t tmem, Ctl &c,
                                               const TreeArgs &a) {
    if (elect_one()) {
        constexpr uint32_t fmt = kF16 ? umma::kFmtF16 : umma::kFmtBF16;
        constexpr uint32_t idesc_s = umma::instr_desc_f16(128, 128, fmt, 0);  // K is K-major
        constexpr uint32_t idesc_o = umma::instr_desc_f16(128, 128, fmt, 1);  // V is MN-major
        // (an operand's other buffer, atom or step: its address field moved on)
        const uint64_t q_desc = umma::smem_desc_kmajor_sw128(saddr(sq));
        const uint64_t k_desc = umma::smem_desc_kmajor_sw128(saddr(sk), kGroup);
        const uint64_t v_desc = umma::smem_desc_mnmajor_sw128(saddr(sv), kChunk, kGroup);
        Walk ws = c.walk, wp = c.walk;
        Piece p;
        // the scores' piece, its items and those done, key tiles before the next; and the product's
        int sn = -1, s_items = 0, s_at = 0, s_two = 0, n = -1, items = 0, at = 0, two = 0;
        uint32_t kt = 0, vt = 0;
        bool more = true;
#pragma unroll 1
        for (uint32_t x = 0;; ++x) {  // the product of item x - 2, then the scores of item x
            const uint32_t h = x & 1, parity = (x >> 1) & 1;
            if (x >= 2) {
                if (at == items) {
                    if (!next(a, c, wp, p)) break;
                    ++n;
                    two = p.rt - 1;
                    items = (p.j1 - p.j0) << two;
                    at = 0;
                    // the first products of a piece overwrite O: the previous piece's read-out must be done
                    if (n > 0 && !lane_wait(&c.o_free, (n - 1) & 1, c, a)) break;
                }
                if (!lane_wait(&c.p_full[h], parity ^ 1, c, a)) break;  // P, and V (see the softmax)
                tc_fence_after();
                const uint32_t stage = vt % kStages;
                // P of keys 16k..16k+15: 8 columns; those of keys 64.. begin where their scores did
                const uint32_t pcol = tmem + h * 128, ocol = pcol + kOCol, add = at >= 2;
                const uint64_t vd = v_desc + stage * (kTileBytes >> 4);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    mma_ts(ocol, pcol + k / 4 * 64 + k % 4 * 8, vd + static_cast<uint64_t>(k * (2 * kGroup >> 4)), idesc_o,
                           k ? 1u : add);
                ++at;
                if (!two || (at & 1) == 0) {  // the tile's last item
                    commit(&c.v_empty[stage]);
                    ++vt;
                }
                if (at == items) commit(&c.o_ready);  // the piece's O is complete
            }
            if (more && s_at == s_items) {
                more = next(a, c, ws, p);
                if (more) {
                    ++sn;
                    s_two = p.rt - 1;
                    s_items = (p.j1 - p.j0) << s_two;
                    s_at = 0;
                    const int b = a.paired ? 0 : sn & 1;
                    if (!lane_wait(&c.q_full[b], (a.paired ? sn : sn >> 1) & 1, c, a)) break;
                }
            }
            if (more) {
                const uint32_t stage = kt % kStages;
                if (!lane_wait(&c.k_full[stage], (kt / kStages) & 1, c, a)) break;
                tc_fence_after();
                const int buf = a.paired ? (s_two ? s_at & 1 : 0) : sn & 1;
                const uint64_t qd = q_desc + buf * (kTileBytes >> 4), kd = k_desc + stage * (kTileBytes >> 4);
#pragma unroll
                for (int k = 0; k < 8; ++k)  // (16 of the 64 columns of an atom are 32 bytes)
                    mma_ss(tmem + h * 128, qd + k / 4 * (kAtom >> 4) + k % 4 * 2, kd + k / 4 * (kChunk >> 4) + k % 4 * 2,
                           idesc_s, k != 0);
                commit(&c.s_full[h]);
                ++s_at;
                if (!s_two || (s_at & 1) == 0) {
                    commit(&c.k_empty[stage]);
                    ++kt;
                }
                if (s_at == s_items) commit(&c.q_empty[a.paired ? 0 : sn & 1]);
            }
        }
        commit(&c.mma_done);
        drain(&c.mma_done, 0);
    }
    __syncwarp();
}

__device__ __forceinline__ void st_global_v8(float *to, const uint32_t *v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ void ld_global_v8(const float *from, float (&v)[8]) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                 : "l"(from)
                 : "memory");
}
// A partial result lies in groups of 8 columns, each for all rows: a warp writes and reads 1024 bytes together.
__device__ __forceinline__ float *part_at(const TreeArgs &a, int64_t slot, int group, int row) {
    return a.part_o + ((slot * (kD / 8) + group) * tree::kRows + row) * 8;
}
// Eight columns of an output row.
template <bool kF16>
__device__ __forceinline__ void store_out(uint64_t to, const float (&o)[8]) {
    *reinterpret_cast<uint4 *>(to) = make_uint4(pack16<kF16>(o[0], o[1]), pack16<kF16>(o[2], o[3]), pack16<kF16>(o[4], o[5]),
                                                pack16<kF16>(o[6], o[7]));
}
// Columns [ch, ch + 32) of row r: to the output row, whole sectors where rows lie on their bounds, or to a partial result.
template <bool kF16>
__device__ __forceinline__ void store_columns(const TreeArgs &a, int64_t slot, uint64_t row, int r, int ch, bool whole,
                                              const uint32_t (&o)[32]) {
    if (!whole) {
#pragma unroll
        for (int u = 0; u < 4; ++u) st_global_v8(part_at(a, slot, ch / 8 + u, r), o + 8 * u);
        return;
    }
    uint32_t y[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) y[u] = pack16<kF16>(__uint_as_float(o[2 * u]), __uint_as_float(o[2 * u + 1]));
    if (a.sectors) {
        st_global_v8(reinterpret_cast<float *>(row + 2 * ch), y);
        st_global_v8(reinterpret_cast<float *>(row + 2 * ch + 32), y + 8);
    } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            *reinterpret_cast<uint4 *>(row + 2 * ch + 16 * u) = make_uint4(y[4 * u], y[4 * u + 1], y[4 * u + 2], y[4 * u + 3]);
    }
}

// Read-out of piece n, as its half's warps noted it (d): of a pair each half its own row tile, else each half
// 64 columns of both accumulators.
template <bool kF16>
__device__ __forceinline__ void read_out(uint32_t tmem, int q, int lane, uint32_t h, int n, const Noted &d, Ctl &c, const TreeArgs &a) {
    const int r = q * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(q * 32) << 16;
    const int tok = prefix::quotient(r, a.s.by_group), g = r - tok * a.s.group;
    const Piece &p = d.p;
    const uint32_t x0 = d.x0;
    const int two = p.rt - 1, items = (p.j1 - p.j0) << two, first = (h ^ x0) & 1;
    const int i = (2 * p.p + (two ? first : 0)) * a.s.tokens + tok;
    const bool live = tok < a.s.tokens && i < p.q.count, any = __any_sync(kFull, live);
    const bool both = !two && items > 1;
    const int only = two ? h : x0 & 1;  // the half that has the (other) sums
    if (any) {
        const bool whole = p.part < 0;
        const int head = p.h * a.s.group + g;
        const int64_t slot = (2ll * blockIdx.x + max(p.part, 0)) * 2 + (two ? first : 0);
        const uint64_t row = reinterpret_cast<uint64_t>(a.out) + 2 * (p.s * a.out_seq + i * a.out_token + head * a.out_head);
        const float2 e = c.ml[n % kMlSlots][both ? 0 : only][r];
        const float2 f = both ? c.ml[n % kMlSlots][1][r] : make_float2(-INFINITY, 0.f);
        const float mx = fmaxf(e.x, f.x), mr = mx == -INFINITY ? 0.f : mx;
        float w0 = e.y == 0.f ? 0.f : ex2(e.x - mr), w1 = f.y == 0.f ? 0.f : ex2(f.x - mr);
        const float total = w0 * e.y + w1 * f.y;  // (NaN stays)
        if (whole) {
            const float inv = total == 0.f ? 0.f : __fdividef(1.f, total);
            w0 *= inv;
            w1 *= inv;
        }
        // (what has no weight may hold anything, NaN too: its bits are cleared)
        const uint32_t keep0 = w0 == 0.f ? 0u : ~0u, keep1 = w1 == 0.f ? 0u : ~0u;
        const uint32_t at0 = tmem + lane_off + kOCol + (both ? 0 : only * 128), at1 = tmem + lane_off + kOCol + 128;
        // 32 columns at a time, of a pair all four quarters, else two with both halves' sums (one body for all,
        // for the instruction cache: read-outs of 16 rows took 3 us)
        const int from = two ? 0 : static_cast<int>(h) * 64, to = two ? 128 : from + 64;
#pragma unroll 1
        for (int ch = from; ch < to; ch += 32) {
            uint32_t o[32], o1[32];
            tmem_ld32_async(at0 + ch, o);
            tmem_ld32_async(at1 + ch, o1);
            tmem_wait_dep(o);
            tmem_wait_dep(o1);
#pragma unroll
            for (int b = 0; b < 32; ++b)
                o[b] = __float_as_uint(__uint_as_float(o[b] & keep0) * w0 + __uint_as_float(o1[b] & keep1) * w1);
            if (live) store_columns<kF16>(a, slot, row, r, ch, whole, o);
        }
        if (live && (two || h == 0)) {
            if (!whole)
                a.part_ml[slot * tree::kRows + r] = make_float2(mx, total);
            else if (a.lse)
                a.lse[(static_cast<int64_t>(p.s) * a.s.n_q + i) * a.n_heads + head] =
                    total == 0.f ? -INFINITY : (mx + log2f(total)) * kLn2;
        }
    }
    if (p.part == 1 && h == 0 && q == 0 && lane == 0) {
        // the unit's other tiles follow the range's end
        const int last = tree::cta_of(c.ranges, c.range_end + p.to_last);
        a.cut[blockIdx.x] = Cut{last - static_cast<int>(blockIdx.x) + 1, static_cast<int>(blockIdx.x), p.s, p.h, p.p, p.q.count, {0, 0}};
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&c.o_free);
}

// Whether a phase of a barrier is over, without a wait; all lanes, on the same answer.
__device__ __forceinline__ bool done_already(uint64_t *bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(saddr(bar)), "r"(parity)
        : "memory");
    return __all_sync(kFull, done != 0);
}

// Softmax and read-out of half h; this thread's row is TMEM lane r of its item's row tile. A piece is read
// out after the half's first item of the next one where the item's scores are there: the piece's last
// product takes as long. (Read out at once: 64 sequences of 32 tokens 86 us instead of 83. After the first
// item always: 128 sequences of one token, 32/8 heads, contexts 20 to 1500, 84 -> 100.)
template <bool kF16>
__device__ __forceinline__ void softmax(uint32_t tmem, int q, int lane, uint32_t h, uint8_t *sv, Ctl &c, const TreeArgs &a) {
    const int r = q * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(q * 32) << 16;
    const uint32_t sbuf = tmem + lane_off + h * 128, obuf = tmem + lane_off + kOCol + h * 128;
    const int tok = prefix::quotient(r, a.s.by_group);  // the row's token in the tile
    Walk w = c.walk;
    Piece p{};
    uint32_t x0 = 0, kt0 = 0;  // items and key tiles of the pieces before
    Noted &noted = c.noted[h * 4 + q];
    bool ok = true, pending = false;
#pragma unroll 1
    for (int n = 0;; ++n) {
        const bool have = next(a, c, w, p);
        if (!have && !pending) break;
        const int two = p.rt - 1, items = have ? (p.j1 - p.j0) << two : 0;
        const int first = (h ^ x0) & 1;                       // the half's first item
        const int i = (2 * p.p + (two ? first : 0)) * a.s.tokens + tok;  // the row's query
        const bool live = tok < a.s.tokens && i < p.q.count;
        const bool any = __any_sync(kFull, live);
        const uint32_t *mask_row = a.s.chain ? nullptr : a.mask + (static_cast<int64_t>(p.s) * a.s.n_q + (live ? i : 0)) * a.words;
        float m = kF16 ? -INFINITY : 0.f, l = 0.f;
        int it = first;
#pragma unroll 1
        do {
            if (it < items && (!pending || done_already(&c.s_full[h], ((x0 + it) >> 1) & 1))) {
                const uint32_t x = x0 + it, kt = kt0 + (it >> two);
                const int key = (p.j0 + (it >> two)) * tree::kRows;
                if (!warp_wait(&c.s_full[h], (x >> 1) & 1, c, a)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                if (any) {
                    // Keys that a row does not see take no weight: a word of 32 keys at a time, quarters in which some
                    // row of the warp has such keys are masked and written back. (Rows that are not stored need
                    // no mask.)
                    const uint32_t bad = c.bad[kt % 4];
                    bool sees = live;
                    if (bad || key + tree::kRows > p.q.len - p.q.count) {
                        uint32_t some = 0, hit = 0;
#pragma unroll 1
                        for (int k = 0; k < tree::kRows; k += 32) {
                            uint32_t word = ~0u;
                            if (live) word = a.s.chain ? tree::chain_bits(p.q, i, key + k)
                                                       : tree::mask_bits(p.q, key + k, [&](int y) { return mask_row[y]; });
                            some |= word;
                            if (bad)
#pragma unroll 1
                                for (int b = 0; b < 32; b += 8)  // (a copy is 8 tokens at least)
                                    if (bad >> ((k + b) >> a.copies.copy_log) & 1u) hit |= word >> b & 0xffu;
                            if (!__any_sync(kFull, word != ~0u)) continue;
                            uint32_t s0[32];
                            tmem_ld32_async(sbuf + k, s0);
                            tmem_wait_dep(s0);
#pragma unroll
                            for (int b = 0; b < 32; ++b)
                                if (!(word >> b & 1u)) s0[b] = __float_as_uint(-INFINITY);
                            tmem_st32_u(sbuf + k, s0);
                        }
                        tmem_wait_st();
                        if (live && hit) l = NAN;  // a page of this row's keys does not exist: NaN
                        sees = live && some != 0 && !hit;
                    }
                    // P = 2^(s c - m) with the row's present reference m, 0 at first; the sum tells whether m was
                    // good enough (P and the sums far from the ends of their types' ranges: for fp16 P, m is
                    // within 2^15 of the largest so far). If not, m becomes the tile's largest score and P is
                    // computed again: P is kept in registers until then, for it overwrites scores.
                    const f2 cc = pack2(a.c, a.c);
                    bool raise = kF16 && m == -INFINITY && sees;
#pragma unroll 1
                    for (int round = 0; round < 2; ++round) {
                        if (__any_sync(kFull, raise)) {
                            float mx8[8];
#pragma unroll
                            for (int b = 0; b < 8; ++b) mx8[b] = -INFINITY;
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
                            // the warp rescales its O together (tcgen05.ld / st are warp-wide), rows without need by
                            // 1. The half's previous product is done: S of this item was issued after it.
                            if (__any_sync(kFull, f != 1.f)) {
#pragma unroll 1
                                for (int ch = 0; ch < 8; ++ch) {
                                    uint32_t o[16];
                                    tmem_ld16_async(obuf + ch * 16, o);
                                    tmem_wait_dep(o);
#pragma unroll
                                    for (int b = 0; b < 16; ++b) o[b] = __float_as_uint(__uint_as_float(o[b]) * f);
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
                        raise = sees && (!(l0 < kMostWeight) || (!kF16 && l == 0.f && l0 < kLeastWeight));
                        if (round == 0 && __any_sync(kFull, raise)) continue;
                        l += l0;
                        tmem_st32_u(sbuf, pk);
                        tmem_st32_u(sbuf + 64, pk2);
                        break;
                    }
                    tmem_wait_st();
                }
                if (it + 2 >= items) c.ml[n % kMlSlots][h][r] = make_float2(l == 0.f ? -INFINITY : m, l);
                // V has to be there, too: the issuer then has one wait less. Where the sequence ends in this tile,
                // the rows of its last page past the end are cleared (later pages' are zeros), by the row
                // tile whose product comes first.
                const int end = p.q.len - key, stop = min(tree::kRows, ((p.q.len + (1 << a.s.page_log) - 1) >> a.s.page_log << a.s.page_log) - key);
                const bool clears = end < stop && (!two || (it & 1) == 0);
                if (clears || q == 0) {
                    const uint32_t stage = kt % kStages;
                    if (!(ok = warp_wait(&c.v_full[stage], (kt / kStages) & 1, c, a))) break;
                    if (clears) {
                        uint8_t *vb = sv + stage * kTileBytes;
#pragma unroll 1
                        for (int y = r; y < (stop - max(end, 0)) * 16; y += 128) {  // 8 16-byte units in each of two chunks
                            const int token = max(end, 0) + (y >> 4);
                            st_shared_v4(saddr(vb + token / 8 * kGroup + (y & 8 ? kChunk : 0) + token % 8 * 128 + (y & 7) * 16),
                                         make_uint4(0, 0, 0, 0));
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&c.p_full[h]);
                it += 2;
            }
            if (pending) {
                if (!(ok = warp_wait(&c.o_ready, (n - 1) & 1, c, a))) break;
                tc_fence_after();
                read_out<kF16>(tmem, q, lane, h, n - 1, noted, c, a);
                pending = false;
            }
        } while (it < items);
        if (!ok) break;
        if (have) {
            __syncwarp();
            if (lane == 0) noted = Noted{p, x0};
            __syncwarp();
            pending = true;
            x0 += items;
            kt0 += p.j1 - p.j0;
        }
    }
}

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                          const __grid_constant__ CUtensorMap tm_v, const TreeArgs a) {
    extern __shared__ uint8_t dyn_smem[];
    __shared__ Ctl c;
    const int warp = __shfl_sync(kFull, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    uint8_t *base = dyn_smem + ((1024u - (saddr(dyn_smem) & 1023u)) & 1023u);
    uint8_t *sq = base;                       // Q buffers
    uint8_t *sk = sq + kQBufs * kTileBytes;   // K stages
    uint8_t *sv = sk + kStages * kTileBytes;  // V stages
    if (threadIdx.x == 0) {
        for (int b = 0; b < 2; ++b) {
            mbar_init(&c.q_full[b], 1);
            mbar_init(&c.q_empty[b], 1);
            mbar_init(&c.k_full[b], 1);
            mbar_init(&c.k_empty[b], 1);
            mbar_init(&c.v_full[b], 1);
            mbar_init(&c.v_empty[b], 1);
            mbar_init(&c.s_full[b], 1);
            mbar_init(&c.p_full[b], 4);  // a half's four warps
        }
        mbar_init(&c.o_ready, 1);
        mbar_init(&c.o_free, 8);
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
    if (threadIdx.x == 0) a.cut[blockIdx.x].parts = 0;
    find_range(a, c);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = c.tmem_base;
    if (warp == 0 || warp == 2)
        produce(warp == 0, warp == 0 ? &tm_k : &tm_v, &tm_q, warp == 0 ? sk : sv, sq, lane, c, a);
    else if (warp == 1)
        issue_products<kF16>(sq, sk, sv, tmem, c, a);
    else if (warp >= 4)
        softmax<kF16>(tmem, warp & 3, lane, (warp >> 2) - 1, sv, c, a);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && c.abort_flag) flag_error(a.err, RPS_DEVERR_TIMEOUT);
    if (warp == 1) tmem_dealloc(tmem, kTmemCols);
}

// ---------------------------------------------------------------- joining the parts of cut units
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;
constexpr int kAhead = 2;                        // parts in flight
constexpr int kJoinCols = 16, kJoinGroups = kJoinCols / 8;  // columns of a warp

struct Joined {
    float m, l, o[kJoinCols];
};
__device__ __forceinline__ void join(Joined &x, float m, float l, const float (&o)[kJoinCols]) {
    const float mm = fmaxf(x.m, m), mr = mm == -INFINITY ? 0.f : mm;
    const float f = ex2(x.m - mr), g = ex2(m - mr);
    x.m = mm;
    x.l = x.l * f + l * g;
#pragma unroll
    for (int b = 0; b < kJoinCols; ++b) x.o[b] = x.o[b] * f + o[b] * g;
}

// Block (cut, some of its rows and columns): a warp takes 32 rows and 16 columns of the cut's unit, of
// `split` warps each one takes parts w, w + split, .... The cuts are those of the CTAs' entries that
// have parts, in order: there are no more than units, so no block is started in vain for each CTA
// (2 sequences, 16 units, context 28000: 19456 blocks, most of them empty, took 20 us).
template <bool kF16>
__global__ void __launch_bounds__(kJoinThreads, 4) tree_combine_kernel(const TreeArgs a, int ctas, int split) {
    __shared__ Joined others[kJoinWarps][32];
    __shared__ int found[kJoinWarps];
    __shared__ Cut cut;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    static_assert(kMaxCtas <= kJoinThreads, "an entry a thread");
    if (threadIdx.x == 0) cut.parts = 0;
    pdl_wait();
    pdl_launch_next();
    // (a call that gave up may not have written its entries: the parts are kept inside the workspace)
    const auto sane = [&](const Cut &x, int cta) { return x.parts > 0 && x.cta == cta && x.parts <= ctas - cta; };
    if (static_cast<int>(gridDim.x) == ctas) {  // a block for each CTA
        if (threadIdx.x == 0) cut = a.cut[blockIdx.x];
        __syncthreads();
        if (!sane(cut, blockIdx.x)) return;
    } else {
        Cut mine{};
        if (static_cast<int>(threadIdx.x) < ctas) mine = a.cut[threadIdx.x];
        const bool is = sane(mine, threadIdx.x);
        const uint32_t in_warp = __ballot_sync(kFull, is);
        if (lane == 0) found[warp] = __popc(in_warp);
        __syncthreads();
        int rank = __popc(in_warp & ((1u << lane) - 1));
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) rank += w < warp ? found[w] : 0;
        if (is && rank == static_cast<int>(blockIdx.x)) cut = mine;
        __syncthreads();
        if (cut.parts == 0) return;
    }
    // the warp's task: its 32 rows (of up to 256), its 16 columns
    const int task = blockIdx.y * (kJoinWarps / split) + warp / split, which = warp % split;
    const int group = task % (kD / kJoinCols) * kJoinGroups, row2 = task / (kD / kJoinCols) * 32 + lane;
    const int rt = row2 >> 7, row = row2 & 127;
    const int t = prefix::quotient(row, a.s.by_group), i = (2 * cut.p + rt) * a.s.tokens + t;
    const bool there = rt < 2 && t < a.s.tokens && i < cut.count;
    Joined x;
    x.m = -INFINITY;
    x.l = 0.f;
#pragma unroll
    for (int b = 0; b < kJoinCols; ++b) x.o[b] = 0.f;
    if (there) {
#pragma unroll 1
        for (int p = which; p < cut.parts; p += split * kAhead) {
            float2 ml[kAhead];
            float o[kAhead][kJoinCols];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int pp = min(p + u * split, cut.parts - 1);
                // the first part of a unit ends its CTA's range, the others begin theirs
                const int64_t slot = (2ll * (cut.cta + pp) + (pp == 0 ? 1 : 0)) * 2 + rt;
                ml[u] = a.part_ml[slot * tree::kRows + row];
#pragma unroll
                for (int g = 0; g < kJoinGroups; ++g)
                    ld_global_v8(part_at(a, slot, group + g, row), *reinterpret_cast<float(*)[8]>(&o[u][8 * g]));
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (p + u * split < cut.parts) join(x, ml[u].x, ml[u].y, o[u]);
        }
    }
    if (split > 1) {
        others[warp][lane] = x;
        __syncthreads();
        if (which) return;
#pragma unroll 1
        for (int w = 1; w < split; ++w) {
            const Joined y = others[warp + w][lane];
            join(x, y.m, y.l, y.o);
        }
    }
    if (!there) return;
    const int head = cut.h * a.s.group + row - t * a.s.group;
    const float inv = x.l == 0.f ? 0.f : 1.f / x.l;
    const uint64_t to = reinterpret_cast<uint64_t>(a.out) + 2 * (cut.s * a.out_seq + i * a.out_token + head * a.out_head + group * 8);
#pragma unroll
    for (int b = 0; b < kJoinCols; ++b) x.o[b] *= inv;
#pragma unroll
    for (int g = 0; g < kJoinGroups; ++g) store_out<kF16>(to + 16 * g, *reinterpret_cast<float(*)[8]>(&x.o[8 * g]));
    if (a.lse && group == 0)
        a.lse[(static_cast<int64_t>(cut.s) * a.s.n_q + i) * a.n_heads + head] =
            x.l == 0.f ? -INFINITY : (x.m + log2f(x.l)) * kLn2;
}

// ---------------------------------------------------------------- host
std::mutex g_tree_mutex;
bool g_tree_ready[64] = {};
int g_tree_sms[64] = {};

rps_status tree_setup(int *sms) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RPS_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g_tree_mutex);
    if (!g_tree_ready[dev]) {
        if (cudaDeviceGetAttribute(&g_tree_sms[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return RPS_ERR_CUDA;
        for (auto k : {tree_attention_kernel<false>, tree_attention_kernel<true>})
            if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess)
                return RPS_ERR_CUDA;
        g_tree_ready[dev] = true;
    }
    *sms = std::min(g_tree_sms[dev], kMaxCtas);
    return RPS_OK;
}

// Shape of a call, with the limits that keep its counts in 32 bits.
rps_status check_tree_shape(const rps_kv_cache *kv, int32_t n_q, int32_t n_heads, int32_t chain, Shape *s) {
    const rps_status st = check_kv_cache(kv);
    if (st != RPS_OK) return st;
    if (n_q < 1 || n_heads < 1 || n_heads % kv->n_heads) return RPS_ERR_INVALID_ARG;
    if (n_heads / kv->n_heads > RPS_KV_MAX_GROUP || n_q > RPS_TREE_MAX_TOKENS) return RPS_ERR_UNSUPPORTED;
    *s = tree::make_shape(kv->n_req * kv->n_branch, n_q, kv->n_heads, n_heads / kv->n_heads, kv->page_size, kv->n_pages,
                          kv->max_pages, chain);
    return RPS_OK;
}

}  // namespace
}  // namespace rps

using namespace rps;

extern "C" size_t rps_tree_attention_workspace_bytes(const rps_kv_cache *kv, int32_t n_q, int32_t n_heads) {
    Shape s;
    if (check_tree_shape(kv, n_q, n_heads, 0, &s) != RPS_OK) return 0;
    return tree::workspace_at(0, sizeof(Cut), kD).bytes;
}

extern "C" rps_status rps_tree_attention_fwd(const rps_tree_attention *p, const rps_kv_cache *kv, void *d_ws, size_t ws_bytes,
                                             rps_stream_t stream) {
    if (!p || !p->q || !p->out) return RPS_ERR_INVALID_ARG;
    TreeArgs a;
    std::memset(&a, 0, sizeof a);
    rps_status st = check_tree_shape(kv, p->n_q, p->n_heads, p->mask == nullptr, &a.s);
    if (st != RPS_OK) return st;
    if (p->layer < 0 || p->layer >= kv->n_layers) return RPS_ERR_INVALID_ARG;
    if (!(p->scale > 0.f) || !std::isfinite(p->scale)) return RPS_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p->q) % 16 || reinterpret_cast<uintptr_t>(p->out) % 16) return RPS_ERR_INVALID_ARG;
    const int64_t ext[3] = {p->n_heads, p->n_q, a.s.n_seq};
    const int64_t qs[3] = {p->q_head_stride, p->q_token_stride, p->q_seq_stride};
    const int64_t os[3] = {p->out_head_stride, p->out_token_stride, p->out_seq_stride};
    for (int i = 0; i < 3; ++i)
        if (ext[i] > 1 && (qs[i] <= 0 || os[i] <= 0 || qs[i] % 8 || os[i] % 8)) return RPS_ERR_INVALID_ARG;
    const tree::Workspace w = tree::workspace_at(reinterpret_cast<uintptr_t>(d_ws), sizeof(Cut), kD);
    if (!d_ws || reinterpret_cast<uintptr_t>(d_ws) % tree::kBaseAlign || ws_bytes < w.bytes) return RPS_ERR_INVALID_ARG;
    int sms = 0;
    if ((st = tree_setup(&sms)) != RPS_OK) return st;
    const Encoder encode = tensor_map_encoder();
    if (!encode || !(a.err = device_error_word())) return RPS_ERR_CUDA;

    const bool f16 = kv->dtype == RPS_F16;
    const uint32_t qbox[3] = {static_cast<uint32_t>(a.s.group), static_cast<uint32_t>(a.s.tokens), 1};
    CUtensorMap tq, tk, tv;
    if ((st = make_map(encode, &tq, p->q, f16, kD, ext, qs, qbox)) != RPS_OK) return st;
    if ((st = map_pages(encode, &tk, &tv, kv, p->layer, std::min(a.s.page_log, 7), a.copies)) != RPS_OK) return st;
    a.table = kv->table;
    a.len = kv->len;
    a.count = p->n_tok;
    a.mask = p->mask;
    a.words = (p->n_q + 31) / 32;
    a.n_heads = p->n_heads;
    a.out = p->out;
    a.out_seq = a.s.n_seq > 1 ? os[2] : 0;
    a.out_token = p->n_q > 1 ? os[1] : 0;
    a.out_head = p->n_heads > 1 ? os[0] : 0;
    a.lse = p->lse;
    a.c = p->scale * kLog2e;
    a.paired = p->n_q > a.s.tokens;
    a.sectors = (reinterpret_cast<uintptr_t>(p->out) | static_cast<uintptr_t>(2 * (a.out_seq | a.out_token | a.out_head))) % 32 == 0;
    char *ws = static_cast<char *>(d_ws);
    a.cut = reinterpret_cast<Cut *>(ws + w.cut);
    a.part_ml = reinterpret_cast<float2 *>(ws + w.ml);
    a.part_o = reinterpret_cast<float *>(ws + w.o);
    a.tries = static_cast<uint32_t>(std::min<uint64_t>((ring_wait_limit_ns() + 999) / 1000, 1u << 30));

    // CTAs: as many as there can be key tiles
    const int64_t tiles = ((static_cast<int64_t>(a.s.max_pages) << a.s.page_log) + tree::kRows - 1) / tree::kRows;
    const int64_t units = static_cast<int64_t>(a.s.n_seq) * a.s.heads * a.s.pairs;
    // Where units are no more than CTAs and cannot be long, none is cut, and there is nothing to join: one launch
    // (one sequence, 32 heads, 16 drafted of 344 tokens: 11.0 to 11.8 us with two, 8.9 to 9.7 with one, by the inputs).
    a.few = units <= std::min(sms, kThreads);  // (so there are no more sequences)
    a.whole = a.few && tiles <= kWholeTiles;
    const int grid = static_cast<int>(std::min<int64_t>(a.whole ? units : units * tiles, sms));
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (launch_pdl(f16 ? tree_attention_kernel<true> : tree_attention_kernel<false>, dim3(grid), dim3(kThreads), kSmemBytes, s,
                   tq, tk, tv, a) != cudaSuccess)
        return RPS_ERR_CUDA;
    if (a.whole) return RPS_OK;
    // a cut unit has about grid / units parts, and there are no more cuts than units: a block for each,
    // and for each 32 rows and 16 columns a warp, or several where the parts are many
    int split = 1;
    while (split < kJoinWarps && units * 2 * kAhead * split < grid) split *= 2;
    const int rows = a.paired ? 2 * tree::kRows : a.s.tokens * a.s.group;
    const int tasks = (rows + 31) / 32 * (kD / kJoinCols), per = kJoinWarps / split;
    return launch_pdl(f16 ? tree_combine_kernel<true> : tree_combine_kernel<false>,
                      dim3(static_cast<unsigned>(std::min<int64_t>(units, grid)), (tasks + per - 1) / per), dim3(kJoinThreads), 0,
                      s, a, grid, split) == cudaSuccess
               ? RPS_OK
               : RPS_ERR_CUDA;
}
