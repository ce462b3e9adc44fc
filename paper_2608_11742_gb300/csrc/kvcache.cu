// kvcache.cu -- pages of the K/V cache: forks, commit, growth with copy on
// write, compaction, copies and writes (rps_kv_*).
//
// The bookkeeping is three integer arrays: page_ref [n_pages] (how many table
// entries hold a page), table [n_seq][max_pages] and len [n_seq] (-1: the
// sequence is absent). A page is free when its count is 0; pages are always
// taken in ascending order and given to the sequences in ascending order, by
// prefix sums, so a call's result does not depend on the order of its atomics.
// Forks and commits of a lookahead step need no order between their sequences: a
// warp each. The other bookkeeping calls are one thread-block cluster (one block of
// it where there is little): its phases are ordered by the cluster barrier, so a call
// that reads what it overwrites needs no second launch, and the counts of the blocks'
// ranges are exchanged through distributed shared memory. The data of copied pages
// follow in a second launch over the whole device. All of these are bound by the
// latency of their dependent accesses (0.6 us each from L2), the data by HBM.
#include <cooperative_groups.h>

#include <algorithm>
#include <cstring>

#include "rps_internal.cuh"

namespace cg = cooperative_groups;

namespace rps {
namespace {

constexpr int kHeadDim = 128;
constexpr int kBookThreads = 1024;
constexpr int kBookWarps = kBookThreads / 32;
constexpr int kCluster = 8;
// Up to these sizes one block does a call's bookkeeping, beyond them a cluster. A cluster's
// barriers cost 1 to 2 us, a block alone has an eighth of the loads in flight. In us, block /
// cluster: reorder (table entries) 234: 3.2 / 3.7, 936: 4.5 / 4.2, 3744: 10.3 / 4.3; growth by two
// pages (pages, or 8 a sequence) 1944: 4.7 / 7.2, 9792: 6.4 / 8.0, but from nothing 14.1 / 9.6;
// compaction (entries and pages) 477: 4.7 / 6.7, 3816: 6.8 / 6.4, 7632: 10.1 / 7.3.
constexpr int kOneReorder = 512, kOneResize = 8192, kOneCompact = 4096;
constexpr int kCopyThreads = 256;
constexpr int kTaskRows = 16;  // rows a warp copies at a time: 4 KB, 8 16-byte loads in flight per lane
constexpr size_t kWsAlign = 256;

struct Book {
    int32_t *ref, *table, *len;
    int32_t n_pages, n_seq, width, ps, log;  // width: table entries of a sequence; ps = 2^log tokens a page
    uint32_t *err;
};

struct CopyHeader {
    int32_t count;    // pages to copy
    int32_t src_off;  // first entry of the source list
};

// Workspace of the calls that change the bookkeeping.
struct KvWorkspace {
    CopyHeader *head;
    int32_t *dst, *src, *used;  // copy list: destination, source, rows (nullptr or -1 pages: skipped)
    int32_t *list;              // free pages in order / source pages by live rank
    int32_t *remap;             // new place of a moved page
    int32_t *snap, *snap_len;   // the rows and lengths a reorder is about to write
    unsigned long long *need;   // per sequence: pages before it (low 32 bits), copies before it (high)
};

size_t ws_align(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }

size_t ws_layout(int64_t n_pages, int64_t n_seq, int64_t width, char *base, KvWorkspace *w) {
    size_t off = 0;
    const auto take = [&](size_t bytes) {
        const size_t at = off;
        off += ws_align(bytes);
        return base ? base + at : nullptr;
    };
    const size_t pages = static_cast<size_t>(n_pages) * 4, seqs = static_cast<size_t>(n_seq) * 4;
    char *head = take(sizeof(CopyHeader)), *dst = take(std::max(pages, seqs)), *src = take(seqs), *used = take(seqs),
         *list = take(pages), *remap = take(pages), *snap = take(seqs * static_cast<size_t>(width)),
         *snap_len = take(seqs), *need = take(seqs * 2);
    if (w) {
        w->head = reinterpret_cast<CopyHeader *>(head);
        w->dst = reinterpret_cast<int32_t *>(dst);
        w->src = reinterpret_cast<int32_t *>(src);
        w->used = reinterpret_cast<int32_t *>(used);
        w->list = reinterpret_cast<int32_t *>(list);
        w->remap = reinterpret_cast<int32_t *>(remap);
        w->snap = reinterpret_cast<int32_t *>(snap);
        w->snap_len = reinterpret_cast<int32_t *>(snap_len);
        w->need = reinterpret_cast<unsigned long long *>(need);
    }
    return off;
}

// ---------------------------------------------------------------- bookkeeping
__device__ __forceinline__ int pages_of(const Book &b, int len) { return len <= 0 ? 0 : ((len - 1) >> b.log) + 1; }

// A sequence's length as it may be used: at most what its table row holds.
__device__ __forceinline__ int checked_len(const Book &b, int len) {
    if (len <= 0) return len < 0 ? -1 : 0;
    if (pages_of(b, len) > b.width) {
        flag_error(b.err, RPS_DEVERR_PAGE);
        return b.width * b.ps;
    }
    return len;
}

__device__ __forceinline__ bool good_page(const Book &b, int p) {
    const bool ok = static_cast<unsigned>(p) < static_cast<unsigned>(b.n_pages);
    if (!ok) flag_error(b.err, RPS_DEVERR_PAGE);
    return ok;
}

// Orders the phases of a bookkeeping call.
__device__ __forceinline__ void book_sync(const cg::cluster_group &cluster) {
    if (cluster.num_blocks() > 1)
        cluster.sync();
    else
        __syncthreads();
}

struct ReorderArgs {
    Book b;
    const int32_t *src_of;
    const int32_t *keep;  // tokens kept, nullptr: all
    KvWorkspace w;
};

// The sequence whose state sequence s takes (-1: none), and how much of it.
__device__ __forceinline__ void source_of(const ReorderArgs &a, int s, int &src, int &keep) {
    keep = INT32_MAX;
    src = a.src_of[s];
    if (src < -1 || src >= a.b.n_seq) {  // the sequence stays as it is
        flag_error(a.b.err, RPS_DEVERR_ROW_INDEX);
        src = s;
    } else if (a.keep) {
        keep = a.keep[s];
    }
}

// A warp per sequence, the rows to be written staged in the workspace between two barriers, for a
// sequence's source may be written by the call itself. 576 sequences of 60 pages: 10 us.
__global__ void __launch_bounds__(kBookThreads, 1) reorder_kernel(const ReorderArgs a) {
    cg::cluster_group cluster = cg::this_cluster();
    const Book &b = a.b;
    const int lane = threadIdx.x & 31;
    const int warp = static_cast<int>(cluster.block_rank()) * kBookWarps + (threadIdx.x >> 5);
    const int warps = static_cast<int>(cluster.num_blocks()) * kBookWarps;
    pdl_wait();
    pdl_launch_next();
    // the old pages are given back, the rows to be written are staged
    for (int s = warp; s < b.n_seq; s += warps) {
        int src, keep;
        source_of(a, s, src, keep);
        const int old_n = pages_of(b, checked_len(b, b.len[s]));
        int len = src < 0 ? -1 : checked_len(b, b.len[src]);
        if (keep < len) len = keep < 0 ? -1 : keep;
        const int n = pages_of(b, len);
        const int32_t *own = b.table + static_cast<int64_t>(s) * b.width;
        for (int i = (src == s ? n : 0) + lane; i < old_n; i += 32)
            if (good_page(b, own[i])) atomicSub(&b.ref[own[i]], 1);
        if (src != s) {
            const int32_t *row = b.table + static_cast<int64_t>(src) * b.width;
            int32_t *to = a.w.snap + static_cast<int64_t>(s) * b.width;
            for (int i = lane; i < n; i += 32) to[i] = row[i];
        }
        if (lane == 0) a.w.snap_len[s] = len;
    }
    book_sync(cluster);
    for (int s = warp; s < b.n_seq; s += warps) {
        int src, keep;
        source_of(a, s, src, keep);
        const int len = a.w.snap_len[s], n = pages_of(b, len);
        int32_t *own = b.table + static_cast<int64_t>(s) * b.width;
        if (src != s) {
            const int32_t *from = a.w.snap + static_cast<int64_t>(s) * b.width;
            for (int i = lane; i < n; i += 32) {
                const int p = from[i];
                own[i] = p;
                if (good_page(b, p)) atomicAdd(&b.ref[p], 1);
            }
        }
        for (int i = n + lane; i < b.width; i += 32) own[i] = -1;
        if (lane == 0) b.len[s] = len;
    }
}

// ---------------------------------------------------------------- a lookahead step's forks and commit
struct BranchArgs {
    Book b;
    const uint8_t *valid;   // fork: [n_req][n_branch - 1]
    const int32_t *ctx;     // fork: tokens kept, nullptr: all
    const int32_t *winner;  // commit (fork if nullptr): [n_req]
    int32_t n_branch;
};

constexpr int kBranchThreads = 128;

// A warp per sequence. Fork: a branch gives its pages back and takes its base's, which nobody
// changes. Commit: the base's warp moves the winner's row to the base (the pages' counts
// stay), the others give their pages back. So no warp reads a row that another writes.
__global__ void __launch_bounds__(kBranchThreads) branch_kernel(const BranchArgs a) {
    const Book &b = a.b;
    const int lane = threadIdx.x & 31, s = blockIdx.x * (kBranchThreads / 32) + (threadIdx.x >> 5);
    if (s >= b.n_seq) return;
    const int q = s / a.n_branch, br = s - q * a.n_branch;
    int32_t *own = b.table + static_cast<int64_t>(s) * b.width;
    pdl_wait();
    pdl_launch_next();
    const int old_len = b.len[s];
    int src = -1, keep = INT32_MAX;  // -1: the sequence ends, s: it stays
    if (a.winner) {
        int w = a.winner[q];
        if (w >= a.n_branch - 1) {  // no such branch: the base stays
            if (br == 0) flag_error(b.err, RPS_DEVERR_ROW_INDEX);
            w = -1;
        }
        if (br == 0) src = w >= 0 ? s + w + 1 : s;
        if (br && br == w + 1) return;  // the base's warp moves it
    } else if (br == 0) {
        src = s;
    } else if (a.valid[static_cast<int64_t>(q) * (a.n_branch - 1) + br - 1]) {
        src = s - br;
        if (a.ctx) keep = a.ctx[q];
    }
    const int old_n = pages_of(b, checked_len(b, old_len));
    int32_t *from = b.table + static_cast<int64_t>(src) * b.width;
    int len = src < 0 ? -1 : checked_len(b, src == s ? old_len : b.len[src]);
    if (keep < len) len = keep < 0 ? -1 : keep;
    const int n = pages_of(b, len), most = max(n, old_n);
    if (src != s) {
        for (int i = lane; i < most; i += 32) {
            const int was = i < old_n ? own[i] : -1, is = i < n ? from[i] : -1;
            if (i < old_n && good_page(b, was)) atomicSub(&b.ref[was], 1);
            own[i] = is;
            if (i >= n) continue;
            const bool good = good_page(b, is);
            if (a.winner)
                from[i] = -1;
            else if (good)
                atomicAdd(&b.ref[is], 1);
        }
        if (lane == 0) {
            b.len[s] = len;
            if (a.winner && src >= 0) b.len[src] = -1;
        }
    }
    for (int i = (src == s ? n : most) + lane; i < b.width; i += 32) own[i] = -1;
    if (a.winner && src >= 0 && src != s)
        for (int i = n + lane; i < b.width; i += 32) from[i] = -1;
}

// Inclusive prefix sum over the block in thread order; the block's total in *total.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long *sums,
                                                         unsigned long long *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long u = __shfl_up_sync(kFull, v, o);
        if (lane >= o) v += u;
    }
    if (lane == 31) sums[warp] = v;
    __syncthreads();
    if (warp == 0) {
        unsigned long long t = sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long u = __shfl_up_sync(kFull, t, o);
            if (lane >= o) t += u;
        }
        sums[lane] = t;
    }
    __syncthreads();
    if (warp) v += sums[warp - 1];
    *total = sums[kBookWarps - 1];
    __syncthreads();  // (sums may be written again)
    return v;
}

// What a block's phases hand on stays in shared memory where it fits, else in the workspace (576
// sequences growing: 15.8 us instead of 16.5).
constexpr int kNearSeqs = 1024;   // sequences of a block
constexpr int kNearPages = 4096;  // free pages
// Up to so many pages a sequence's thread takes or gives back alone, more the warp does together,
// sequence after sequence. Two pages of each of 72 sequences given back: 4.7 us instead of 11.7
// by warps; 24 pages each taken and given back, 7.6 instead of 13.5; 60 each of 9216 sequences,
// alone 107 instead of 79.
constexpr int kFewPages = 32;

struct Counts {
    unsigned long long need;  // of the block's sequences: pages (low 32 bits), copies (high)
    int32_t pages;            // of the block's pages: free ones, or live ones
};

struct ResizeArgs {
    Book b;
    const int32_t *new_len;
    KvWorkspace w;
};

// What a sequence asks for: pages wanted in the low 32 bits, 1 << 32 where its
// shared last page (in `last` then) has to be copied first.
__device__ __forceinline__ unsigned long long wanted(const Book &b, int s, int old_len, int new_len, int &last) {
    if (new_len <= old_len) return 0;
    const int n_old = pages_of(b, old_len);
    unsigned long long need = static_cast<unsigned>(pages_of(b, new_len) - n_old);
    if (old_len > 0 && (old_len & (b.ps - 1))) {
        last = b.table[static_cast<int64_t>(s) * b.width + n_old - 1];
        if (good_page(b, last) && b.ref[last] > 1) need += (1ull << 32) + 1;
    }
    return need;
}

// The length a sequence is to have: one beyond its table row leaves it as it is.
__device__ __forceinline__ int wanted_len(const Book &b, int new_len, int old_len) {
    if (new_len < 0) return -1;
    if (pages_of(b, new_len) > b.width) {
        flag_error(b.err, RPS_DEVERR_PAGE);
        return old_len;
    }
    return new_len;
}

// A sequence of the block: length at first, length it is to have, the last page that it held.
struct Near {
    int32_t old_len, new_len, last;
};

// Growth and shrinking: give back, sum up what is asked for, list the lowest free pages, hand them
// out; the prefix sums give every sequence its part of the list whatever the order of threads. A
// chain of a dozen accesses to L2 and three barriers: 4.2 us for 9 sequences with the empty copy
// launch behind it, 8 for 576 (a cluster), where one thread after another would need each
// sequence's pages to be known before the next.
__global__ void __launch_bounds__(kBookThreads, 1) resize_kernel(const ResizeArgs a) {
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ unsigned long long sums[kBookWarps];
    __shared__ Counts mine;
    __shared__ unsigned long long near_need[kNearSeqs];
    __shared__ Near near_seq[kNearSeqs];
    __shared__ int32_t near_list[kNearPages];
    const Book &b = a.b;
    const int lane = threadIdx.x & 31, rank = cluster.block_rank(), blocks = cluster.num_blocks();
    const int per_s = (b.n_seq + blocks - 1) / blocks;
    const int s0 = min(b.n_seq, rank * per_s), s1 = min(b.n_seq, s0 + per_s);
    const int per_p = (b.n_pages + blocks - 1) / blocks;
    const int p0 = min(b.n_pages, rank * per_p), p1 = min(b.n_pages, p0 + per_p);
    const bool near = per_s <= kNearSeqs;  // the block's sequences are kept in shared memory
    pdl_wait();
    pdl_launch_next();
    const auto lengths = [&](int s) {
        Near x;
        x.old_len = checked_len(b, b.len[s]);
        x.new_len = wanted_len(b, a.new_len[s], x.old_len);
        x.last = -1;
        return x;
    };
    // 1. pages past a shorter sequence's end go back
    for (int at = s0; at < s1; at += kBookThreads) {
        const int s = at + threadIdx.x;
        Near x{0, 0, -1};
        if (s < s1) {
            x = lengths(s);
            if (near) near_seq[s - s0] = x;
        }
        const int held = pages_of(b, x.old_len), count = x.new_len < x.old_len ? held - pages_of(b, x.new_len) : 0;
        const auto give = [&](int seq, int entry) {
            int32_t *at = b.table + static_cast<int64_t>(seq) * b.width + entry;
            const int p = *at;
            if (good_page(b, p)) atomicSub(&b.ref[p], 1);
            *at = -1;
        };
        if (count <= kFewPages)
            for (int i = 1; i <= count; ++i) give(s, held - i);
        for (uint32_t m = __ballot_sync(kFull, count > kFewPages); m; m &= m - 1) {
            const int who = __ffs(m) - 1, n = __shfl_sync(kFull, count, who), h = __shfl_sync(kFull, held, who);
            for (int i = 1 + lane; i <= n; i += 32) give(s - lane + who, h - i);
        }
        if (x.new_len < x.old_len) {
            b.len[s] = x.new_len;
            if (near) near_seq[s - s0].old_len = x.new_len;
        }
    }
    book_sync(cluster);
    // 2. what the block's sequences ask for, and the free ones of the block's pages (of a block
    // alone they are counted as they are listed)
    unsigned long long carry = 0, total;
    for (int at = s0; at < s1; at += kBookThreads) {
        const int s = at + threadIdx.x;
        unsigned long long need = 0;
        int last = -1;
        if (s < s1) {
            const Near x = near ? near_seq[s - s0] : lengths(s);
            need = wanted(b, s, x.old_len, x.new_len, last);
        }
        const unsigned long long upto = block_scan(need, sums, &total);
        if (s < s1) {
            (near ? near_need[s - s0] : a.w.need[s]) = carry + upto - need;
            if (near) near_seq[s - s0].last = last;
        }
        carry += total;
    }
    unsigned long long need_before = 0, need_all = carry;
    int free_before = 0, free_all = 0;
    if (blocks > 1) {
        int free_here = 0;
        for (int p = p0 + threadIdx.x; p < p1; p += kBookThreads) free_here += b.ref[p] <= 0;
        block_scan(free_here, sums, &total);
        if (threadIdx.x == 0) {
            mine.need = carry;
            mine.pages = static_cast<int32_t>(total);
        }
        cluster.sync();
        need_all = 0;
        for (int r = 0; r < blocks; ++r) {
            const Counts *c = cluster.map_shared_rank(&mine, r);
            if (r < rank) {
                need_before += c->need;
                free_before += c->pages;
            }
            need_all += c->need;
            free_all += c->pages;
        }
    }
    // 3. the lowest free pages, in order, as many as are asked for; a thread takes four neighbours
    const int wish = static_cast<int>(min(need_all & 0xffffffffull, static_cast<unsigned long long>(INT32_MAX)));
    int32_t *list = blocks == 1 && wish <= kNearPages ? near_list : a.w.list;
    for (int at = p0; at < p1 && free_before < wish; at += 4 * kBookThreads) {
        const int p = at + 4 * threadIdx.x;
        uint32_t is_free = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (p + i < p1 && b.ref[p + i] <= 0) is_free |= 1u << i;
        const int count = __popc(is_free);
        int to = free_before + static_cast<int>(block_scan(count, sums, &total)) - count;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (is_free >> i & 1u) {
                if (to < wish) list[to] = p + i;
                ++to;
            }
        free_before += static_cast<int>(total);
    }
    if (blocks == 1) free_all = free_before;  // (all that there are, or as many as are asked for)
    book_sync(cluster);  // (the list is written, and every block has read every count)
    // 4. each sequence takes its pages, a thread's own where they are few; the copy list
    for (int at = s0; at < s1; at += kBookThreads) {
        const int s = at + threadIdx.x;
        int first = 0, count = 0;  // table entries that take pages
        int64_t from = 0;          // their first page in the list
        Near x{0, 0, -1};
        if (s < s1) x = near ? near_seq[s - s0] : lengths(s);
        if (x.new_len > x.old_len) {
            // (counts of pages change while this phase runs: what is wanted is the difference to the next sequence)
            const auto need_of = [&](int i) { return need_before + (i >= s1 ? carry : near ? near_need[i - s0] : a.w.need[i]); };
            const unsigned long long off = need_of(s), next = need_of(s + 1);
            const bool cow = (next >> 32) != (off >> 32);
            const bool fits = (next & 0xffffffffull) <= static_cast<unsigned long long>(free_all);
            const int n_old = pages_of(b, x.old_len);
            from = static_cast<int64_t>(off & 0xffffffffull);
            if (!fits) flag_error(b.err, RPS_DEVERR_NO_PAGES);
            if (cow) {
                const int e = static_cast<int>(off >> 32);
                if (!near) x.last = b.table[static_cast<int64_t>(s) * b.width + n_old - 1];
                a.w.src[e] = fits ? x.last : -1;
                a.w.dst[e] = fits ? list[from] : -1;
                a.w.used[e] = x.old_len & (b.ps - 1);
                if (fits) atomicSub(&b.ref[x.last], 1);
            }
            if (fits) {
                first = n_old - (cow ? 1 : 0);
                count = pages_of(b, x.new_len) - first;
                b.len[s] = x.new_len;
            }
        }
        const auto take = [&](int seq, int entry, int64_t i) {
            const int p = list[i];
            b.table[static_cast<int64_t>(seq) * b.width + entry] = p;
            b.ref[p] = 1;
        };
        if (count <= kFewPages)
            for (int i = 0; i < count; ++i) take(s, first + i, from + i);
        for (uint32_t m = __ballot_sync(kFull, count > kFewPages); m; m &= m - 1) {  // more: the warp together
            const int who = __ffs(m) - 1, n = __shfl_sync(kFull, count, who), f = __shfl_sync(kFull, first, who);
            const int64_t l = __shfl_sync(kFull, from, who);
            for (int i = lane; i < n; i += 32) take(s - lane + who, f + i, l + i);
        }
    }
    if (rank == 0 && threadIdx.x == 0) {
        a.w.head->count = static_cast<int32_t>(need_all >> 32);
        a.w.head->src_off = 0;
    }
}

struct CompactArgs {
    Book b;
    int32_t *n_live;
    KvWorkspace w;
};

// Both lists by one pass of prefix sums over the counts, then the counts move, then the table
// entries are renamed: 10 us for 8000 pages and 576 sequences, beside 160 for the pages' data.
__global__ void __launch_bounds__(kBookThreads, 1) compact_kernel(const CompactArgs a) {
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ unsigned long long sums[kBookWarps];
    __shared__ Counts mine;
    const Book &b = a.b;
    const int lane = threadIdx.x & 31, rank = cluster.block_rank(), blocks = cluster.num_blocks();
    const int warp = rank * kBookWarps + (threadIdx.x >> 5), warps = blocks * kBookWarps;
    pdl_wait();
    pdl_launch_next();
    const int per_p = (b.n_pages + blocks - 1) / blocks;
    const int p0 = min(b.n_pages, rank * per_p), p1 = min(b.n_pages, p0 + per_p);
    unsigned long long total;
    int live_here = 0;
    for (int p = p0 + threadIdx.x; p < p1; p += kBookThreads) live_here += b.ref[p] > 0;
    block_scan(live_here, sums, &total);
    int before = 0, n_live = static_cast<int>(total);
    if (blocks > 1) {
        if (threadIdx.x == 0) mine.pages = n_live;
        cluster.sync();
        n_live = 0;
        for (int r = 0; r < blocks; ++r) {
            const int c = cluster.map_shared_rank(&mine, r)->pages;
            if (r < rank) before += c;
            n_live += c;
        }
    }
    // The i-th free page below n_live takes the i-th live page from n_live on. Live
    // pages go into `list` by their rank among all live ones, so the sources are its
    // entries from the number of live pages below n_live on.
    for (int at = p0; at < p1; at += kBookThreads) {
        const int p = at + threadIdx.x;
        const bool live = p < p1 && b.ref[p] > 0;
        const int upto = static_cast<int>(block_scan(live, sums, &total));
        const int live_before = before + upto - (live ? 1 : 0);
        if (p < p1) {
            if (live && p >= n_live) a.w.list[live_before] = p;
            if (!live && p < n_live) a.w.dst[p - live_before] = p;
            if (!live && p >= n_live) a.w.remap[p] = p;  // (a table entry whose page has a count of 0 stays)
            if (p == n_live) {
                a.w.head->src_off = live_before;
                a.w.head->count = n_live - live_before;
            }
        }
        before += static_cast<int>(total);
    }
    if (rank == 0 && threadIdx.x == 0) {
        if (a.n_live) *a.n_live = n_live;
        if (n_live == b.n_pages) a.w.head->src_off = a.w.head->count = 0;
    }
    book_sync(cluster);
    const int moved = a.w.head->count, src_off = a.w.head->src_off;
    for (int i = rank * kBookThreads + threadIdx.x; i < moved; i += blocks * kBookThreads) {
        const int src = a.w.list[src_off + i], dst = a.w.dst[i];
        a.w.remap[src] = dst;
        b.ref[dst] = b.ref[src];
        b.ref[src] = 0;
    }
    book_sync(cluster);
    for (int s = warp; s < b.n_seq; s += warps) {
        const int n = pages_of(b, checked_len(b, b.len[s]));
        int32_t *row = b.table + static_cast<int64_t>(s) * b.width;
        for (int i = lane; i < n; i += 32) {
            const int p = row[i];
            if (good_page(b, p) && p >= n_live) row[i] = a.w.remap[p];
        }
    }
}

// ---------------------------------------------------------------- data
struct PageData {
    uint4 *k, *v;
    int64_t layer, page, head, token;  // strides in 16-byte units
};

struct CopyArgs {
    PageData from, to;
    const int32_t *src, *dst, *used;  // used == nullptr: whole pages
    const CopyHeader *head;           // nullptr: `count` pages from the lists' first entries
    int32_t count, n_from, n_to, layers, heads, ps;
    uint32_t *err;
};

// A warp copies up to 16 rows (a token of a head each, 256 bytes) at a time, half a warp to a
// row: 8 loads of 16 bytes a lane in flight. Bound by HBM: 1000 pages of 32 tokens, 8 heads, 4
// layers (524 MB read, as much written) 161 us, 96 % of a plain copy's bandwidth; three blocks an
// SM (with four, 64 registers a thread, the loads no longer stay together: 168).
__global__ void __launch_bounds__(kCopyThreads, 3) copy_kernel(const CopyArgs a) {
    const int lane = threadIdx.x & 31;
    pdl_wait();
    pdl_launch_next();
    const int count = a.head ? a.head->count : a.count, src_off = a.head ? a.head->src_off : 0;
    const int blocks = (a.ps + kTaskRows - 1) / kTaskRows;  // of a page's tokens
    const int per = a.layers * 2 * a.heads * blocks;        // tasks of a page
    const int64_t task = static_cast<int64_t>(blockIdx.x) * (kCopyThreads / 32) + (threadIdx.x >> 5);
    const int64_t step = static_cast<int64_t>(gridDim.x) * (kCopyThreads / 32);
    int e = static_cast<int>(task / per), t = static_cast<int>(task - static_cast<int64_t>(e) * per);
    const int64_t step_e = step / per;
    const int step_t = static_cast<int>(step - step_e * per);
    // (the entry of the next task is on its way while a task's rows are)
    const auto entry = [&](int64_t i, int &src, int &dst, int &used) {
        src = dst = -1;
        used = 0;
        if (i >= count) return;
        src = a.src[src_off + i];
        dst = a.dst[i];
        used = a.used ? a.used[i] : a.ps;
    };
    int src, dst, used;
    entry(e, src, dst, used);
    for (int64_t ee = e; ee < count;) {
        int x = t;
        const int block = x % blocks;
        x /= blocks;
        const int head = x % a.heads;
        x /= a.heads;
        const int which = x & 1, layer = x >> 1;
        const int rows = min(kTaskRows, used - block * kTaskRows);
        const bool skip = a.used && src < 0;  // (a copy that found no page)
        const bool ok = static_cast<unsigned>(src) < static_cast<unsigned>(a.n_from) &&
                        static_cast<unsigned>(dst) < static_cast<unsigned>(a.n_to) && rows > 0;
        if (!ok && !skip && rows > 0) flag_error(a.err, RPS_DEVERR_PAGE);
        const int row0 = block * kTaskRows + (lane >> 4);
        const uint4 *s = (which ? a.from.v : a.from.k) + layer * a.from.layer + src * a.from.page + head * a.from.head +
                         row0 * a.from.token + (lane & 15);
        uint4 *d = (which ? a.to.v : a.to.k) + layer * a.to.layer + dst * a.to.page + head * a.to.head +
                   row0 * a.to.token + (lane & 15);
        uint4 v[kTaskRows / 2];
#pragma unroll
        for (int i = 0; i < kTaskRows / 2; ++i)
            if (ok && 2 * i + (lane >> 4) < rows) v[i] = __ldcs(s + 2 * i * a.from.token);
        ee += step_e;
        t += step_t;
        if (t >= per) {
            t -= per;
            ++ee;
        }
        entry(ee, src, dst, used);
#pragma unroll
        for (int i = 0; i < kTaskRows / 2; ++i)
            if (ok && 2 * i + (lane >> 4) < rows) d[2 * i * a.to.token] = v[i];
    }
}

struct WriteArgs {
    Book b;
    PageData to;  // of one layer
    const uint4 *k, *v;
    int64_t seq, token, head;  // strides of the new rows, in 16-byte units
    int32_t n_new, heads, blocks;  // blocks: of one sequence's keys (or values)
    uint32_t by_heads;             // ceil(2^32 / heads)
};

constexpr int kWriteRows = 512;  // rows (token, head) of a block

// A block writes up to 512 of a sequence's new key (or value) rows: first the place of each
// token, looked up once, then the rows, 16 of a warp in flight. (Places looked up row by
// row, 16 rows a warp: 576 x 32 tokens of 32 heads 120 us; so 96, 93 % of a copy's bandwidth.)
__global__ void __launch_bounds__(kCopyThreads) write_kernel(const WriteArgs a) {
    __shared__ int64_t place[kWriteRows];  // of a token's first head, -1: none
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int group = blockIdx.x / a.blocks, block = blockIdx.x - group * a.blocks;
    const int s = group >> 1, row0 = block * kWriteRows, rows = min(kWriteRows, a.n_new * a.heads - row0);
    const int tok0 = row0 / a.heads, skip = row0 - tok0 * a.heads;  // the first row's token and head
    const int toks = (skip + rows - 1) / a.heads + 1;
    pdl_wait();
    pdl_launch_next();
    const int len = checked_len(a.b, a.b.len[s]);
    if (len < 0) return;
    const int32_t *row = a.b.table + static_cast<int64_t>(s) * a.b.width;
    const int log = a.b.log;
    for (int i = threadIdx.x; i < toks; i += kCopyThreads) {
        const int pos = len - a.n_new + tok0 + i;
        int64_t at = -1;
        if (pos >= 0) {
            const int p = row[pos >> log];
            if (good_page(a.b, p)) {
                if (a.b.ref[p] > 1)  // others read this page too
                    flag_error(a.b.err, RPS_DEVERR_SHARED);
                else
                    at = p * a.to.page + (pos & (a.b.ps - 1)) * a.to.token;
            }
        }
        place[i] = at;
    }
    __syncthreads();
    const uint4 *from = ((group & 1) ? a.v : a.k) + s * a.seq + tok0 * a.token + (lane & 15);
    uint4 *to = ((group & 1) ? a.to.v : a.to.k) + (lane & 15);
    constexpr int kDeep = kTaskRows / 2;
    for (int r0 = warp * kTaskRows; r0 < rows; r0 += kCopyThreads / 32 * kTaskRows) {
        uint4 v[kDeep];
        int64_t at[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const int r = r0 + 2 * i + (lane >> 4);
            at[i] = -1;
            if (r >= rows) continue;
            const int x = r + skip, tok = a.heads == 1 ? x : static_cast<int>(__umulhi(x, a.by_heads)), head = x - tok * a.heads;
            v[i] = __ldcs(from + tok * a.token + head * a.head);
            at[i] = place[tok];
            if (at[i] >= 0) at[i] += head * a.to.head;
        }
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
            if (at[i] >= 0) to[at[i]] = v[i];
    }
}

// ---------------------------------------------------------------- host
// One block, or a cluster of eight.
template <typename Args>
rps_status launch_book(void (*kernel)(Args), const Args &a, bool one_block, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    const int blocks = one_block ? 1 : kCluster;
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(kBookThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = blocks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess ? RPS_OK : RPS_ERR_CUDA;
}

bool strides_ok(int64_t extent, int64_t stride) { return extent == 1 || (stride > 0 && stride % 8 == 0); }

// Sizes and layout of the pages.
rps_status check_pages(const rps_kv_cache *kv) {
    if (!kv || !kv->k || !kv->v) return RPS_ERR_INVALID_ARG;
    if (kv->dtype != RPS_BF16 && kv->dtype != RPS_F16) return RPS_ERR_INVALID_ARG;
    if (kv->n_layers < 1 || kv->n_pages < 1 || kv->n_heads < 1 || kv->page_size < 1) return RPS_ERR_INVALID_ARG;
    if (kv->head_dim != kHeadDim) return RPS_ERR_UNSUPPORTED;
    if (kv->page_size < RPS_KV_MIN_PAGE || kv->page_size > RPS_KV_MAX_PAGE || (kv->page_size & (kv->page_size - 1)))
        return RPS_ERR_UNSUPPORTED;
    if (kv->n_layers > RPS_KV_MAX_LAYERS || kv->n_heads > RPS_KV_MAX_HEADS) return RPS_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(kv->k) % 16 || reinterpret_cast<uintptr_t>(kv->v) % 16) return RPS_ERR_INVALID_ARG;
    if (!strides_ok(kv->n_layers, kv->layer_stride) || !strides_ok(kv->n_pages, kv->page_stride) ||
        !strides_ok(kv->n_heads, kv->head_stride) || !strides_ok(kv->page_size, kv->token_stride))
        return RPS_ERR_INVALID_ARG;
    return RPS_OK;
}

rps_status check_cache(const rps_kv_cache *kv, Book *b) {
    rps_status st = check_pages(kv);
    if (st != RPS_OK) return st;
    if (!kv->page_ref || !kv->table || !kv->len) return RPS_ERR_INVALID_ARG;
    if (kv->n_req < 1 || kv->n_branch < 1 || kv->max_pages < 1) return RPS_ERR_INVALID_ARG;
    const int64_t n_seq = static_cast<int64_t>(kv->n_req) * kv->n_branch;
    if (n_seq > RPS_KV_MAX_SEQ || static_cast<int64_t>(kv->max_pages) * kv->page_size > INT32_MAX / 2 ||
        n_seq * kv->max_pages > INT32_MAX || kv->n_pages > INT32_MAX / 2)
        return RPS_ERR_UNSUPPORTED;
    if (b) {
        b->ref = kv->page_ref;
        b->table = kv->table;
        b->len = kv->len;
        b->n_pages = kv->n_pages;
        b->n_seq = static_cast<int32_t>(n_seq);
        b->width = kv->max_pages;
        b->ps = kv->page_size;
        b->log = 0;
        while ((1 << b->log) < b->ps) ++b->log;
        b->err = nullptr;
    }
    return RPS_OK;
}

rps_status prepare(const rps_kv_cache *kv, void *d_ws, size_t ws_bytes, Book *b, KvWorkspace *w) {
    rps_status st = check_cache(kv, b);
    if (st != RPS_OK) return st;
    if (!d_ws || reinterpret_cast<uintptr_t>(d_ws) % 16 ||
        ws_bytes < ws_layout(b->n_pages, b->n_seq, b->width, nullptr, nullptr))
        return RPS_ERR_INVALID_ARG;
    ws_layout(b->n_pages, b->n_seq, b->width, static_cast<char *>(d_ws), w);
    b->err = device_error_word();
    return b->err ? RPS_OK : RPS_ERR_CUDA;
}

PageData page_data(const rps_kv_cache *kv) {
    PageData d;
    d.k = static_cast<uint4 *>(kv->k);
    d.v = static_cast<uint4 *>(kv->v);
    d.layer = kv->n_layers > 1 ? kv->layer_stride / 8 : 0;
    d.page = kv->n_pages > 1 ? kv->page_stride / 8 : 0;
    d.head = kv->n_heads > 1 ? kv->head_stride / 8 : 0;
    d.token = kv->token_stride / 8;
    return d;
}

rps_status launch_copy(const rps_kv_cache *from, const rps_kv_cache *to, const int32_t *src, const int32_t *dst,
                       const int32_t *used, const CopyHeader *head, int32_t count, int64_t most, uint32_t *err,
                       cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms < 1) return RPS_ERR_CUDA;
    CopyArgs a;
    std::memset(&a, 0, sizeof a);
    a.from = page_data(from);
    a.to = page_data(to);
    a.src = src;
    a.dst = dst;
    a.used = used;
    a.head = head;
    a.count = count;
    a.n_from = from->n_pages;
    a.n_to = to->n_pages;
    a.layers = to->n_layers;
    a.heads = to->n_heads;
    a.ps = to->page_size;
    a.err = err;
    const int64_t tasks = most * a.layers * 2 * a.heads * ((a.ps + kTaskRows - 1) / kTaskRows);
    const int64_t blocks = std::min<int64_t>((tasks + kCopyThreads / 32 - 1) / (kCopyThreads / 32), sms * 8);
    return launch_pdl(copy_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kCopyThreads), 0, stream, a) == cudaSuccess
               ? RPS_OK
               : RPS_ERR_CUDA;
}

rps_status launch_branches(const rps_kv_cache *kv, const uint8_t *valid, const int32_t *ctx, const int32_t *winner,
                           void *d_ws, size_t ws_bytes, cudaStream_t stream) {
    BranchArgs a;
    std::memset(&a, 0, sizeof a);
    KvWorkspace w;  // (taken and checked like the other calls', not used)
    const rps_status st = prepare(kv, d_ws, ws_bytes, &a.b, &w);
    if (st != RPS_OK) return st;
    a.valid = valid;
    a.ctx = ctx;
    a.winner = winner;
    a.n_branch = kv->n_branch;
    const int per = kBranchThreads / 32;
    return launch_pdl(branch_kernel, dim3((a.b.n_seq + per - 1) / per), dim3(kBranchThreads), 0, stream, a) == cudaSuccess
               ? RPS_OK
               : RPS_ERR_CUDA;
}

}  // namespace

rps_status check_kv_cache(const rps_kv_cache *kv) { return check_cache(kv, nullptr); }

}  // namespace rps

using namespace rps;

extern "C" {

size_t rps_kv_workspace_bytes(const rps_kv_cache *kv) {
    Book b;
    if (check_cache(kv, &b) != RPS_OK) return 0;
    return ws_layout(b.n_pages, b.n_seq, b.width, nullptr, nullptr);
}

rps_status rps_kv_reorder(const rps_kv_cache *kv, const int32_t *d_src, const int32_t *d_keep, void *d_ws,
                          size_t ws_bytes, rps_stream_t stream) {
    if (!d_src) return RPS_ERR_INVALID_ARG;
    ReorderArgs a;
    std::memset(&a, 0, sizeof a);
    const rps_status st = prepare(kv, d_ws, ws_bytes, &a.b, &a.w);
    if (st != RPS_OK) return st;
    a.src_of = d_src;
    a.keep = d_keep;
    return launch_book(reorder_kernel, a, static_cast<int64_t>(a.b.n_seq) * a.b.width <= kOneReorder, reinterpret_cast<cudaStream_t>(stream));
}

rps_status rps_kv_fork_branches(const rps_kv_cache *kv, const uint8_t *d_branch_valid, const int32_t *d_ctx_len,
                                void *d_ws, size_t ws_bytes, rps_stream_t stream) {
    if (!d_branch_valid || !kv || kv->n_branch < 2) return RPS_ERR_INVALID_ARG;
    return launch_branches(kv, d_branch_valid, d_ctx_len, nullptr, d_ws, ws_bytes, reinterpret_cast<cudaStream_t>(stream));
}

rps_status rps_kv_commit(const rps_kv_cache *kv, const int32_t *d_winner, void *d_ws, size_t ws_bytes,
                         rps_stream_t stream) {
    if (!d_winner) return RPS_ERR_INVALID_ARG;
    return launch_branches(kv, nullptr, nullptr, d_winner, d_ws, ws_bytes, reinterpret_cast<cudaStream_t>(stream));
}

rps_status rps_kv_resize(const rps_kv_cache *kv, const int32_t *d_new_len, void *d_ws, size_t ws_bytes,
                         rps_stream_t stream) {
    if (!d_new_len) return RPS_ERR_INVALID_ARG;
    ResizeArgs a;
    std::memset(&a, 0, sizeof a);
    rps_status st = prepare(kv, d_ws, ws_bytes, &a.b, &a.w);
    if (st != RPS_OK) return st;
    a.new_len = d_new_len;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if ((st = launch_book(resize_kernel, a, std::max(8 * a.b.n_seq, a.b.n_pages) <= kOneResize, s)) != RPS_OK) return st;
    return launch_copy(kv, kv, a.w.src, a.w.dst, a.w.used, a.w.head, 0, a.b.n_seq, a.b.err, s);
}

rps_status rps_kv_compact(const rps_kv_cache *kv, int32_t *d_n_live, void *d_ws, size_t ws_bytes, rps_stream_t stream) {
    CompactArgs a;
    std::memset(&a, 0, sizeof a);
    rps_status st = prepare(kv, d_ws, ws_bytes, &a.b, &a.w);
    if (st != RPS_OK) return st;
    a.n_live = d_n_live;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if ((st = launch_book(compact_kernel, a, static_cast<int64_t>(a.b.n_seq) * a.b.width + a.b.n_pages <= kOneCompact, s)) != RPS_OK) return st;
    return launch_copy(kv, kv, a.w.list, a.w.dst, nullptr, a.w.head, 0, (static_cast<int64_t>(kv->n_pages) + 1) / 2,
                       a.b.err, s);
}

rps_status rps_kv_copy_pages(const rps_kv_cache *from, const rps_kv_cache *to, const int32_t *d_src,
                             const int32_t *d_dst, int32_t n, rps_stream_t stream) {
    rps_status st = check_pages(from);
    if (st != RPS_OK || (st = check_pages(to)) != RPS_OK) return st;
    if (n < 0 || (n > 0 && (!d_src || !d_dst))) return RPS_ERR_INVALID_ARG;
    if (from->dtype != to->dtype || from->n_layers != to->n_layers || from->n_heads != to->n_heads ||
        from->page_size != to->page_size)
        return RPS_ERR_INVALID_ARG;
    if (n == 0) return RPS_OK;
    uint32_t *err = device_error_word();
    if (!err) return RPS_ERR_CUDA;
    return launch_copy(from, to, d_src, d_dst, nullptr, nullptr, n, n, err, reinterpret_cast<cudaStream_t>(stream));
}

rps_status rps_kv_write(const rps_kv_cache *kv, int32_t layer, const void *k_new, const void *v_new, int32_t n_new,
                        int64_t seq_stride, int64_t token_stride, int64_t head_stride, rps_stream_t stream) {
    WriteArgs a;
    std::memset(&a, 0, sizeof a);
    const rps_status st = check_cache(kv, &a.b);
    if (st != RPS_OK) return st;
    if (!k_new || !v_new || layer < 0 || layer >= kv->n_layers || n_new < 1) return RPS_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(k_new) % 16 || reinterpret_cast<uintptr_t>(v_new) % 16) return RPS_ERR_INVALID_ARG;
    if (seq_stride % 8 || token_stride % 8 || head_stride % 8 || seq_stride < 0 || token_stride < 0 || head_stride < 0)
        return RPS_ERR_INVALID_ARG;
    if (static_cast<int64_t>(n_new) * kv->n_heads > INT32_MAX / 2) return RPS_ERR_UNSUPPORTED;
    a.to = page_data(kv);
    a.to.k += layer * a.to.layer;
    a.to.v += layer * a.to.layer;
    a.k = static_cast<const uint4 *>(k_new);
    a.v = static_cast<const uint4 *>(v_new);
    a.seq = seq_stride / 8;
    a.token = token_stride / 8;
    a.head = head_stride / 8;
    a.n_new = n_new;
    a.heads = kv->n_heads;
    a.blocks = (n_new * kv->n_heads + kWriteRows - 1) / kWriteRows;
    // (x * ceil(2^32 / heads) >> 32 is x / heads for x below 512 + heads: the excess is x / 2^32 at most.
    // One head: x itself, which the product would miss)
    a.by_heads = static_cast<uint32_t>(((uint64_t{1} << 32) + kv->n_heads - 1) / kv->n_heads);
    const int64_t grid = 2ll * a.b.n_seq * a.blocks;
    if (grid > INT32_MAX) return RPS_ERR_UNSUPPORTED;
    a.b.err = device_error_word();
    if (!a.b.err) return RPS_ERR_CUDA;
    return launch_pdl(write_kernel, dim3(static_cast<unsigned>(grid)), dim3(kCopyThreads), 0,
                      reinterpret_cast<cudaStream_t>(stream), a) == cudaSuccess
               ? RPS_OK
               : RPS_ERR_CUDA;
}

}  // extern "C"
