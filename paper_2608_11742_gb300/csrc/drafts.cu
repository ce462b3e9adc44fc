// drafts.cu -- drafted tokens of a sequence: from their parents to the masks of what
// they see and their positions (rps_tree_masks), and the keys and values of the
// accepted path to the front of the drafted ones (rps_kv_keep_path).
#include <algorithm>
#include <cstring>

#include "rps_internal.cuh"

namespace rps {
namespace {

// ---------------------------------------------------------------- masks
struct MaskArgs {
    const int32_t *parent, *count, *len;
    uint32_t *mask;
    int32_t *pos;
    int32_t n_tok, words;
    uint32_t *err;
};

// A block per sequence, a thread per token: it walks up to the context. A parent comes
// before its children, so the walk goes through the words of the token's mask from the
// last to the first, and each is written once. Bound by the walk, one dependent access to shared
// memory an ancestor, and by its instructions: in a deep tree each step ends a word in some lane
// of the warp, whose store the others wait for, and a block's 32 warps walk together. 500 trees of up
// to 253 tokens with fans of 2 and 3 (depths about 8): 4.3 us; chains: 1 x 32 tokens 3.2, 1 x 253 36,
// 500 x 253 44, 1 x 1024 190.
__global__ void __launch_bounds__(RPS_TREE_MAX_TOKENS) tree_masks_kernel(const MaskArgs a) {
    __shared__ int32_t parent[RPS_TREE_MAX_TOKENS];
    const int i = threadIdx.x;
    const int64_t s = blockIdx.x;
    pdl_wait();
    pdl_launch_next();
    const int count = a.count ? min(max(a.count[s], 0), a.n_tok) : a.n_tok;
    if (i < count) {
        int p = a.parent[s * a.n_tok + i];
        if (p < -1 || p >= i) {
            flag_error(a.err, RPS_DEVERR_ROW_INDEX);
            p = -1;
        }
        parent[i] = p;
    }
    const int first = a.pos && a.len ? a.len[s] - count : 0;
    __syncthreads();
    if (i >= count) return;
    uint32_t *to = a.mask + (s * a.n_tok + i) * a.words;
    for (int w = a.words - 1; w > i >> 5; --w) to[w] = 0;
    int depth = -1, word = i >> 5;
    uint32_t bits = 0;
    for (int j = i; j >= 0; j = parent[j]) {
        for (; word > j >> 5; --word) {
            to[word] = bits;
            bits = 0;
        }
        bits |= 1u << (j & 31);
        ++depth;
    }
    for (; word >= 0; --word) {
        to[word] = bits;
        bits = 0;
    }
    if (a.pos) a.pos[s * a.n_tok + i] = first + depth;
}

// ---------------------------------------------------------------- kept paths
struct KeepArgs {
    uint4 *k, *v;
    int64_t layer, page, head, token;  // strides in 16-byte units
    const int32_t *table, *len, *ref, *path, *keep, *count;
    int32_t *new_len;
    int32_t n_path, n_q, width, log, n_pages, heads, rows;  // rows: layers x 2 x heads
    uint32_t *err;
};

constexpr int kKeepThreads = 256;
constexpr int kHalves = kKeepThreads / 16;
constexpr int kDeep = 8;  // rows of a half warp in flight

// Block (slice of the layers' heads, sequence): the places of the path's tokens are looked
// up once, then a half warp moves a head's rows, in order and 8 at a time. The path ascends,
// so its d-th entry is d at least: no row is written before it is read. Bound by HBM, by rows of
// 256 bytes scattered over the cache (64 sequences, 32 layers of 8 heads, up to 17 of 64 tokens:
// 27 us, 4.9 TB/s read and written).
__global__ void __launch_bounds__(kKeepThreads) keep_kernel(const KeepArgs a) {
    __shared__ int64_t from[RPS_TREE_MAX_TOKENS], to[RPS_TREE_MAX_TOKENS];
    __shared__ int32_t bad;
    const int64_t s = blockIdx.y;
    if (threadIdx.x == 0) bad = 0;
    pdl_wait();
    pdl_launch_next();
    const int len = a.len[s];
    const int count = a.count ? min(max(a.count[s], 0), a.n_q) : a.n_q;
    const int keep = a.keep[s], ctx = len - count;
    const bool first = blockIdx.x == 0;
    if (len < 0) {
        if (first && threadIdx.x == 0 && a.new_len) a.new_len[s] = -1;
        return;
    }
    const bool sane = keep >= 0 && keep <= min(a.n_path, count) && ctx >= 0 && (len == 0 || (len - 1) >> a.log < a.width);
    __syncthreads();
    if (sane) {
        const int32_t *path = a.path + s * a.n_path, *row = a.table + s * a.width;
        for (int d = threadIdx.x; d < keep; d += kKeepThreads) {
            const int p = path[d];
            if (p >= count || p < 0 || (d > 0 && path[d - 1] >= p)) {
                bad = 1;
                continue;
            }
            const int x = ctx + p, y = ctx + d;
            const int px = row[x >> a.log], py = row[y >> a.log];
            const auto good = [&](int q) { return static_cast<unsigned>(q) < static_cast<unsigned>(a.n_pages); };
            int64_t at = -1;
            if (x == y) {
            } else if (!good(px) || !good(py)) {
                if (first) flag_error(a.err, RPS_DEVERR_PAGE);
            } else if (a.ref[py] > 1) {  // others read this page too
                if (first) flag_error(a.err, RPS_DEVERR_SHARED);
            } else {
                at = py * a.page + (y & ((1 << a.log) - 1)) * a.token;
            }
            from[d] = px * a.page + (x & ((1 << a.log) - 1)) * a.token;
            to[d] = at;
        }
    }
    __syncthreads();
    const bool go = sane && !bad;
    if (first && threadIdx.x == 0) {
        if (!go) flag_error(a.err, RPS_DEVERR_ROW_INDEX);
        if (a.new_len) a.new_len[s] = go ? ctx + keep : len;
    }
    if (!go) return;
    const int half = threadIdx.x >> 4, lane = threadIdx.x & 15;
    for (int r = blockIdx.x * kHalves + half; r < a.rows; r += gridDim.x * kHalves) {
        const int head = r % a.heads, which = r / a.heads & 1, layer = r / a.heads >> 1;
        uint4 *base = (which ? a.v : a.k) + layer * a.layer + head * a.head + lane;
        for (int d0 = 0; d0 < keep; d0 += kDeep) {
            uint4 x[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
                if (d0 + u < keep && to[d0 + u] >= 0) x[u] = base[from[d0 + u]];
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
                if (d0 + u < keep && to[d0 + u] >= 0) base[to[d0 + u]] = x[u];
        }
    }
}

}  // namespace
}  // namespace rps

using namespace rps;

extern "C" {

rps_status rps_tree_masks(const int32_t *d_parent, const int32_t *d_n_tok, const int32_t *d_len, int32_t n_seq, int32_t n_tok,
                          uint32_t *d_mask, int32_t *d_pos, rps_stream_t stream) {
    if (!d_parent || !d_mask || n_seq < 1 || n_tok < 1) return RPS_ERR_INVALID_ARG;
    if (n_tok > RPS_TREE_MAX_TOKENS) return RPS_ERR_UNSUPPORTED;
    MaskArgs a;
    std::memset(&a, 0, sizeof a);
    a.parent = d_parent;
    a.count = d_n_tok;
    a.len = d_len;
    a.mask = d_mask;
    a.pos = d_pos;
    a.n_tok = n_tok;
    a.words = (n_tok + 31) / 32;
    if (!(a.err = device_error_word())) return RPS_ERR_CUDA;
    return launch_pdl(tree_masks_kernel, dim3(static_cast<unsigned>(n_seq)), dim3((n_tok + 31) / 32 * 32), 0,
                      reinterpret_cast<cudaStream_t>(stream), a) == cudaSuccess
               ? RPS_OK
               : RPS_ERR_CUDA;
}

rps_status rps_kv_keep_path(const rps_kv_cache *kv, const int32_t *d_path, const int32_t *d_n_keep, int32_t n_path,
                            const int32_t *d_n_tok, int32_t n_q, int32_t *d_new_len, rps_stream_t stream) {
    const rps_status st = check_kv_cache(kv);
    if (st != RPS_OK) return st;
    if (!d_path || !d_n_keep || n_path < 1 || n_q < 1) return RPS_ERR_INVALID_ARG;
    if (n_path > RPS_TREE_MAX_TOKENS || n_q > RPS_TREE_MAX_TOKENS) return RPS_ERR_UNSUPPORTED;
    KeepArgs a;
    std::memset(&a, 0, sizeof a);
    a.k = static_cast<uint4 *>(kv->k);
    a.v = static_cast<uint4 *>(kv->v);
    a.layer = kv->n_layers > 1 ? kv->layer_stride / 8 : 0;
    a.page = kv->n_pages > 1 ? kv->page_stride / 8 : 0;
    a.head = kv->n_heads > 1 ? kv->head_stride / 8 : 0;
    a.token = kv->token_stride / 8;
    a.table = kv->table;
    a.len = kv->len;
    a.ref = kv->page_ref;
    a.path = d_path;
    a.keep = d_n_keep;
    a.count = d_n_tok;
    a.new_len = d_new_len;
    a.n_path = n_path;
    a.n_q = n_q;
    a.width = kv->max_pages;
    while ((1 << a.log) < kv->page_size) ++a.log;
    a.n_pages = kv->n_pages;
    a.heads = kv->n_heads;
    a.rows = kv->n_layers * 2 * kv->n_heads;
    const int32_t n_seq = kv->n_req * kv->n_branch;
    if (n_seq > 65535) return RPS_ERR_UNSUPPORTED;
    if (!(a.err = device_error_word())) return RPS_ERR_CUDA;
    // a half warp for each head of a layer: fewer blocks with several heads each were slower (64 sequences, 32
    // layers, 8 heads: 2048 blocks 27.4 us, 1216 28.1, 704 30.1)
    const unsigned slices = static_cast<unsigned>(std::min((a.rows + kHalves - 1) / kHalves, 4096));
    return launch_pdl(keep_kernel, dim3(slices, static_cast<unsigned>(n_seq)), dim3(kKeepThreads), 0,
                      reinterpret_cast<cudaStream_t>(stream), a) == cudaSuccess
               ? RPS_OK
               : RPS_ERR_CUDA;
}

}  // extern "C"
