// rope.cu -- the norms of queries and keys for each head and the rotation by their
// positions in one pass over the rows: from tensor to tensor (rps_rope_heads), and
// on the way into the paged K/V cache (rps_kv_append).
//
// For a head x of D elements: y = x w / sqrt(mean(x^2) + eps) where its side has
// weights, else y = x; then each pair (y0, y1) of the first R elements is turned by
// its angle a = 2 pi f t, t the position: A (y0 cos a - y1 sin a), A (y1 cos a + y0 sin a).
// The frequency f of a pair is given in turns per position as a fraction of 2^64, so
// t f modulo 2^64 is the fraction of a turn exactly, whatever the position: what is
// left to fp32 is half a turn at most. All in fp32, rounded once at the end.
//
// Bound by HBM: 4 D bytes a row (16-bit elements read and written once). A lane holds
// 16 elements of a row in two 16-byte units, chosen so that both elements of its
// pairs are its own: in the half layout units l and l + R / 16, else 2l and 2l + 1. A
// warp takes rows of one token, so its 32 lanes compute the token's sines and cosines
// once, and share them through shared memory.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "rps_internal.cuh"

namespace rps {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kPasses = 4;  // rows of a lane in flight
constexpr int kMaxDim = 256;

struct Side {
    const char *src;
    char *dst;
    int64_t src_seq, src_token, src_head, dst_seq, dst_token, dst_head;  // bytes
    int32_t heads;
    const void *weight;  // nullptr: not normed
};

struct RotateArgs {
    Side q, k;
    const uint64_t *turns;
    int32_t R, interleaved;
    float amplitude, eps, inv_d;
    int32_t D, n_tok;
    const int32_t *pos;
    int32_t rows, passes, chunks;  // rows of a token (queries, keys, values), passes of a task, tasks of a token
    int64_t tasks;
    // append: the values, and where keys and values go
    Side v;
    const int32_t *table, *len, *ref, *count;
    int32_t width, page_log, n_pages;
    int64_t page_stride, head_stride, token_stride;  // bytes, of the cache
    uint32_t *err;
};

template <bool kF16>
__device__ __forceinline__ float2 widen(uint32_t x) {
    if (kF16) return __half22float2(*reinterpret_cast<const __half2 *>(&x));
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x));
}
template <bool kF16>
__device__ __forceinline__ uint32_t narrow(float lo, float hi) {
    if (kF16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// Eight elements of a 16-byte unit.
template <bool kF16>
__device__ __forceinline__ void widen8(const uint4 &u, float *x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = widen<kF16>(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
template <bool kF16>
__device__ __forceinline__ uint4 narrow8(const float *x) {
    return make_uint4(narrow<kF16>(x[0], x[1]), narrow<kF16>(x[2], x[3]), narrow<kF16>(x[4], x[5]), narrow<kF16>(x[6], x[7]));
}

__device__ __forceinline__ void turn(float &y0, float &y1, float cs, float sn) {
    const float z0 = y0 * cs - y1 * sn;
    y1 = y1 * cs + y0 * sn;
    y0 = z0;
}

// kLanes lanes to a row (16 elements each), 32 / kLanes rows of a token at a time.
template <bool kF16, int kLanes, bool kPaged>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotateArgs a) {
    __shared__ float2 turned[kWarps][kMaxDim / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kAt = 32 / kLanes;
    const int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
    pdl_wait();
    pdl_launch_next();
    if (task >= a.tasks) return;
    const int64_t x = task / a.chunks;
    const int row0 = static_cast<int>(task - x * a.chunks) * a.passes * kAt + lane / kLanes;
    const int64_t s = x / a.n_tok;
    const int i = static_cast<int>(x - s * a.n_tok);
    int len = 0, count = a.n_tok;
    if (kPaged) {
        len = a.len[s];
        if (a.count) count = min(max(a.count[s], 0), a.n_tok);
        if (len < 0 || i >= count) return;
        if (len > 0 && (len - 1) >> a.page_log >= a.width) {
            if (lane == 0) flag_error(a.err, RPS_DEVERR_PAGE);
            len = a.width << a.page_log;
        }
    }
    const int token = kPaged ? len - count + i : i;
    if (token < 0) return;  // (a row without a place)

    // this lane's 16-byte units of a row
    const int l = lane % kLanes;
    const bool rotates = l < a.R / 16, there = l < a.D / 16;
    const bool halves = rotates && !a.interleaved;
    const int u0 = (halves ? l : 2 * l) * 16, u1 = (halves ? l + a.R / 16 : 2 * l + 1) * 16;
    uint4 raw0[kPasses], raw1[kPasses];
    const auto side_of = [&](int row, int &head) -> const Side & {
        head = row;
        if (row < a.q.heads) return a.q;
        head -= a.q.heads;
        if (!kPaged || head < a.k.heads) return a.k;
        head -= a.k.heads;
        return a.v;
    };
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int row = row0 + p * kAt;
        if (p >= a.passes || row >= a.rows || !there) continue;
        int head;
        const Side &d = side_of(row, head);
        const char *from = d.src + s * d.src_seq + i * d.src_token + head * d.src_head;
        raw0[p] = __ldcs(reinterpret_cast<const uint4 *>(from + u0));
        raw1[p] = __ldcs(reinterpret_cast<const uint4 *>(from + u1));
    }
    // the token's place, and its sines and cosines while the rows are on their way
    int64_t place = -1;
    if (kPaged) {
        const int page = a.table[s * a.width + (token >> a.page_log)];
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.n_pages)) {
            if (lane == 0) flag_error(a.err, RPS_DEVERR_PAGE);
        } else if (a.ref[page] > 1) {  // others read this page too
            if (lane == 0) flag_error(a.err, RPS_DEVERR_SHARED);
        } else {
            place = page * a.page_stride + (token & ((1 << a.page_log) - 1)) * a.token_stride;
        }
    }
    if (a.R) {
        const int64_t t = a.pos ? a.pos[x] : token;
        for (int p = lane; p < a.R / 2; p += 32) {
            const int64_t turn = static_cast<int64_t>(static_cast<uint64_t>(t) * a.turns[p]);
            float sn, cs;
            sincospif(static_cast<float>(turn) * 0x1p-63f, &sn, &cs);
            turned[warp][p] = make_float2(cs * a.amplitude, sn * a.amplitude);
        }
        __syncwarp();
    }
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 f = rotates ? turned[warp][8 * l + j] : make_float2(1.f, 0.f);
        cs[j] = f.x;
        sn[j] = f.y;
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        if (p >= a.passes) break;  // (the same for the whole warp)
        const int row = row0 + p * kAt;
        const bool live = row < a.rows && there;
        int head;
        const Side &d = side_of(row, head);
        const bool value = kPaged && row >= a.q.heads + a.k.heads;
        if (!value) {
            float y[16];
            if (live) {
                widen8<kF16>(raw0[p], y);
                widen8<kF16>(raw1[p], y + 8);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) y[j] = 0.f;
            }
            if (d.weight) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 16; ++j) sum += y[j] * y[j];
                // (the lanes of a row agree on its side)
                const unsigned mask = (kLanes == 32 ? kFull : (1u << kLanes) - 1) << (lane / kLanes * kLanes);
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
                const float r = rsqrtf(sum * a.inv_d + a.eps);
                if (live) {
                    float w[16];
                    widen8<kF16>(*reinterpret_cast<const uint4 *>(static_cast<const char *>(d.weight) + u0), w);
                    widen8<kF16>(*reinterpret_cast<const uint4 *>(static_cast<const char *>(d.weight) + u1), w + 8);
#pragma unroll
                    for (int j = 0; j < 16; ++j) y[j] *= r * w[j];
                }
            }
            // (a loop for each layout: one that picked its elements would put them into local memory)
            if (halves) {
#pragma unroll
                for (int j = 0; j < 8; ++j) turn(y[j], y[j + 8], cs[j], sn[j]);
            } else if (rotates) {
#pragma unroll
                for (int j = 0; j < 8; ++j) turn(y[2 * j], y[2 * j + 1], cs[j], sn[j]);
            }
            raw0[p] = narrow8<kF16>(y);
            raw1[p] = narrow8<kF16>(y + 8);
        }
        if (!live) continue;
        char *to;
        if (kPaged && row >= a.q.heads) {
            if (place < 0) continue;
            to = d.dst + place + head * a.head_stride;
        } else {
            to = d.dst + s * d.dst_seq + i * d.dst_token + head * d.dst_head;
        }
        *reinterpret_cast<uint4 *>(to + u0) = raw0[p];
        *reinterpret_cast<uint4 *>(to + u1) = raw1[p];
    }
}

bool aligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool stride_ok(int64_t extent, int64_t stride) { return extent == 1 || (stride >= 0 && stride % 8 == 0); }

rps_status check_rope(const rps_rope *rope, int32_t head_dim, RotateArgs *a) {
    a->D = head_dim;
    a->inv_d = 1.f / head_dim;
    if (!rope) return RPS_OK;
    if (rope->rotary_dim < 0 || rope->rotary_dim > head_dim) return RPS_ERR_INVALID_ARG;
    if (rope->rotary_dim % 16) return RPS_ERR_UNSUPPORTED;
    if (rope->rotary_dim && (!rope->turns || !std::isfinite(rope->amplitude))) return RPS_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(rope->turns) % 8 || !aligned(rope->q_weight) || !aligned(rope->k_weight))
        return RPS_ERR_INVALID_ARG;
    if ((rope->q_weight || rope->k_weight) && !(rope->eps >= 0.f && std::isfinite(rope->eps))) return RPS_ERR_INVALID_ARG;
    a->turns = rope->turns;
    a->R = rope->rotary_dim;
    a->interleaved = rope->interleaved != 0;
    a->amplitude = rope->amplitude;
    a->eps = rope->eps;
    a->q.weight = rope->q_weight;
    a->k.weight = rope->k_weight;
    return RPS_OK;
}

// One side of a call; strides of dimensions of one are not used.
rps_status check_side(const rps_heads *h, int32_t n_seq, int32_t n_tok, bool with_dst, Side *d) {
    if (!h->src || (with_dst && !h->dst) || h->n_heads < 1) return RPS_ERR_INVALID_ARG;
    if (h->n_heads > RPS_KV_MAX_HEADS * RPS_KV_MAX_GROUP) return RPS_ERR_UNSUPPORTED;
    if (!aligned(h->src) || (with_dst && !aligned(h->dst))) return RPS_ERR_INVALID_ARG;
    if (!stride_ok(n_seq, h->src_seq) || !stride_ok(n_tok, h->src_token) || !stride_ok(h->n_heads, h->src_head))
        return RPS_ERR_INVALID_ARG;
    if (with_dst && ((n_seq > 1 && h->dst_seq <= 0) || (n_tok > 1 && h->dst_token <= 0) || (h->n_heads > 1 && h->dst_head <= 0) ||
                     !stride_ok(n_seq, h->dst_seq) || !stride_ok(n_tok, h->dst_token) || !stride_ok(h->n_heads, h->dst_head)))
        return RPS_ERR_INVALID_ARG;
    d->src = static_cast<const char *>(h->src);
    d->dst = static_cast<char *>(h->dst);
    d->src_seq = n_seq > 1 ? h->src_seq * 2 : 0;
    d->src_token = n_tok > 1 ? h->src_token * 2 : 0;
    d->src_head = h->n_heads > 1 ? h->src_head * 2 : 0;
    d->dst_seq = n_seq > 1 ? h->dst_seq * 2 : 0;
    d->dst_token = n_tok > 1 ? h->dst_token * 2 : 0;
    d->dst_head = h->n_heads > 1 ? h->dst_head * 2 : 0;
    d->heads = h->n_heads;
    return RPS_OK;
}

template <bool kPaged>
rps_status launch_rotate(RotateArgs &a, int32_t n_seq, bool f16, cudaStream_t stream) {
    const int sms = device_sm_count();
    if (sms < 1) return RPS_ERR_CUDA;
    const int lanes = a.D <= 64 ? 4 : a.D <= 128 ? 8 : 16, at = 32 / lanes;
    const int64_t tokens = static_cast<int64_t>(n_seq) * a.n_tok;
    // Few rows are spread over more warps: a warp's rows come one after another.
    const auto chunks = [&](int passes) { return (a.rows + passes * at - 1) / (passes * at); };
    a.passes = kPasses;
    while (a.passes > 1 && tokens * chunks(a.passes) < sms * 8) a.passes /= 2;
    a.chunks = chunks(a.passes);
    a.tasks = tokens * a.chunks;
    const int64_t blocks = (a.tasks + kWarps - 1) / kWarps;
    if (blocks > INT32_MAX) return RPS_ERR_UNSUPPORTED;
    const auto kernel = lanes == 4   ? (f16 ? rotate_kernel<true, 4, kPaged> : rotate_kernel<false, 4, kPaged>)
                        : lanes == 8 ? (f16 ? rotate_kernel<true, 8, kPaged> : rotate_kernel<false, 8, kPaged>)
                                     : (f16 ? rotate_kernel<true, 16, kPaged> : rotate_kernel<false, 16, kPaged>);
    return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, a) == cudaSuccess ? RPS_OK
                                                                                                                : RPS_ERR_CUDA;
}

}  // namespace
}  // namespace rps

using namespace rps;

extern "C" {

uint64_t rps_rope_turns(double radians) {
    if (!std::isfinite(radians)) return 0;
    const double turns = radians / 6.283185307179586476925286766559;
    const double part = turns - std::floor(turns);  // [0, 1]
    const double scaled = std::ldexp(part, 64);
    return scaled >= 18446744073709551616.0 ? 0 : static_cast<uint64_t>(scaled);
}

rps_status rps_rope_heads(const rps_rope *rope, const rps_heads *q, const rps_heads *k, int32_t dtype, int32_t head_dim,
                          int32_t n_seq, int32_t n_tok, const int32_t *d_pos, rps_stream_t stream) {
    if (!rope || !q || n_seq < 1 || n_tok < 1 || head_dim < 1) return RPS_ERR_INVALID_ARG;
    if (dtype != RPS_BF16 && dtype != RPS_F16) return RPS_ERR_INVALID_ARG;
    if (head_dim % 16 || head_dim > kMaxDim) return RPS_ERR_UNSUPPORTED;
    RotateArgs a;
    std::memset(&a, 0, sizeof a);
    rps_status st = check_rope(rope, head_dim, &a);
    if (st != RPS_OK || (st = check_side(q, n_seq, n_tok, true, &a.q)) != RPS_OK) return st;
    if (k && (st = check_side(k, n_seq, n_tok, true, &a.k)) != RPS_OK) return st;
    a.n_tok = n_tok;
    a.pos = d_pos;
    a.rows = a.q.heads + a.k.heads;
    return launch_rotate<false>(a, n_seq, dtype == RPS_F16, reinterpret_cast<cudaStream_t>(stream));
}

rps_status rps_kv_append(const rps_kv_cache *kv, int32_t layer, const rps_rope *rope, const rps_heads *q,
                         const rps_heads *k_new, const rps_heads *v_new, int32_t n_new, const int32_t *d_n_tok,
                         const int32_t *d_pos, rps_stream_t stream) {
    rps_status st = check_kv_cache(kv);
    if (st != RPS_OK) return st;
    if (!k_new || !v_new || layer < 0 || layer >= kv->n_layers || n_new < 1) return RPS_ERR_INVALID_ARG;
    if (k_new->n_heads != kv->n_heads || v_new->n_heads != kv->n_heads) return RPS_ERR_INVALID_ARG;
    RotateArgs a;
    std::memset(&a, 0, sizeof a);
    const int32_t n_seq = kv->n_req * kv->n_branch;
    if ((st = check_rope(rope, kv->head_dim, &a)) != RPS_OK) return st;
    if (q && (st = check_side(q, n_seq, n_new, true, &a.q)) != RPS_OK) return st;
    if ((st = check_side(k_new, n_seq, n_new, false, &a.k)) != RPS_OK || (st = check_side(v_new, n_seq, n_new, false, &a.v)) != RPS_OK)
        return st;
    const int64_t at = kv->n_layers > 1 ? layer * kv->layer_stride * 2 : 0;
    a.k.dst = static_cast<char *>(kv->k) + at;
    a.v.dst = static_cast<char *>(kv->v) + at;
    a.n_tok = n_new;
    a.pos = d_pos;
    a.rows = a.q.heads + 2 * kv->n_heads;
    a.table = kv->table;
    a.len = kv->len;
    a.ref = kv->page_ref;
    a.count = d_n_tok;
    a.width = kv->max_pages;
    while ((1 << a.page_log) < kv->page_size) ++a.page_log;
    a.n_pages = kv->n_pages;
    a.page_stride = kv->n_pages > 1 ? kv->page_stride * 2 : 0;
    a.head_stride = kv->n_heads > 1 ? kv->head_stride * 2 : 0;
    a.token_stride = kv->token_stride * 2;
    if (!(a.err = device_error_word())) return RPS_ERR_CUDA;
    return launch_rotate<true>(a, n_seq, kv->dtype == RPS_F16, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
