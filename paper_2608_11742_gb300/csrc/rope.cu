// rope.cu -- the norms of queries and keys for each head and the rotation by their
// positions in one pass over the rows: from tensor to tensor (rps_rope_heads), and
// on the way into the paged K/V cache (rps_kv_append).
//
// For a head x of D elements: y = x w / sqrt(mean(x^2) + eps) where its side has
// weights, else y = x; then each pair (y0, y1) of the first R elements is turned by
// its angle a = 2 pi f t, t the position: A (y0 cos a - y1 sin a), A (y1 cos a + y0 sin a).
// The frequency f of a pair is given in turns per position as a fraction of 2^64, so
// t f modulo 2^64 is the fraction of a turn exactly, whatever the position. It is cut to 32 bits, half a turn
// at most (1.5e-9 of a radian), and rounded to fp32's 24: 1e-7 of a radian at most near half a turn, relative to
// smaller angles 2^-24, as every fp32 step behind it. All in fp32, rounded once at the end.
//
// Bound by HBM: 4 D bytes a row (16-bit elements read and written once), as long as a pass
// of a warp over 1024 bytes takes less than about 170 instructions (at twice as many, 576 x 32
// tokens of 96 rows, half of them there, took 106 us). A lane holds 16 elements of a row
// in two 16-byte units, chosen so that both elements of its pairs are its own: in the half
// layout units l and l + R / 16, else 2l and 2l + 1. A warp takes rows of one token and one
// side, so its lanes compute the token's sines and cosines once, share them through shared
// memory, and multiply them with the weights once:
//   z0 = r ((w0 cos) y0 - (w1 sin) y1),  z1 = r ((w1 cos) y1 + (w0 sin) y0),  r = 1 / sqrt(..),
// two pairs to an instruction (packed fp32). A lane whose elements are not rotated leaves the sines' products
// out (0 times an infinity is NaN), and without a norm its elements go through bit for bit.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "rps_internal.cuh"
#include "tc_device.cuh"

namespace rps {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kAhead = 4;  // passes of a warp in shared memory
constexpr int kMaxDim = 256;
constexpr int kFullWarps = 24;  // of an SM

// (A division of 32 bits where they are enough.)
__device__ __forceinline__ int64_t divide(int64_t x, int32_t d) {
    return x >> 32 ? x / d : static_cast<int64_t>(static_cast<uint32_t>(x) / static_cast<uint32_t>(d));
}

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
    int32_t passes_q, passes_k, passes_all;  // passes of a token's queries, of its keys, of all its rows
    int32_t passes, chunks;                  // of a task; tasks of a token
    int64_t tasks;
    // append: the values, and where keys and values go
    Side v;
    const int32_t *table, *len, *ref, *count;
    int32_t width, page_log, n_pages;
    int64_t page_stride, head_stride, token_stride;  // bytes, of the cache
    uint32_t *err;
};

// Two 16-bit elements as fp32.
template <bool kF16>
__device__ __forceinline__ float2 widen(uint32_t x) {
    if (kF16) return __half22float2(*reinterpret_cast<const __half2 *>(&x));
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
// A lane's 16 elements as the first and the second ones of its eight pairs, two pairs to an f2:
// unit by unit, or (interleaved) the even and the odd ones of both units.
template <bool kF16>
__device__ __forceinline__ void widen16(const uint4 &u, const uint4 &v, bool interleaved, f2 (&y0)[4], f2 (&y1)[4]) {
    const uint32_t a[4] = {u.x, u.y, u.z, u.w}, b[4] = {v.x, v.y, v.z, v.w};
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = widen<kF16>(i < 2 ? a[2 * i] : b[2 * i - 4]), g = widen<kF16>(i < 2 ? a[2 * i + 1] : b[2 * i - 3]);
            y0[i] = pack2(f.x, g.x);
            y1[i] = pack2(f.y, g.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = widen<kF16>(a[i]), g = widen<kF16>(b[i]);
            y0[i] = pack2(f.x, f.y);
            y1[i] = pack2(g.x, g.y);
        }
    }
}
template <bool kF16>
__device__ __forceinline__ void narrow16(const f2 (&y0)[4], const f2 (&y1)[4], bool interleaved, uint4 &u, uint4 &v) {
    uint32_t a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float p, q, r, s;
        unpack2(y0[i], p, q);
        unpack2(y1[i], r, s);
        a[i] = interleaved ? pack16<kF16>(p, r) : pack16<kF16>(p, q);
        b[i] = interleaved ? pack16<kF16>(q, s) : pack16<kF16>(r, s);
    }
    if (interleaved) {
        u = make_uint4(a[0], b[0], a[1], b[1]);
        v = make_uint4(a[2], b[2], a[3], b[3]);
    } else {
        u = make_uint4(a[0], a[1], a[2], a[3]);
        v = make_uint4(b[0], b[1], b[2], b[3]);
    }
}

// c += a b in the lanes where `is` (a predicate; as a branch: 45.5 us instead of 44.2 for the append below)
__device__ __forceinline__ void fma2_if(f2 &c, f2 a, f2 b, bool is) {
    asm("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\t@p fma.rn.f32x2 %0, %1, %2, %0;\n\t}"
        : "+l"(c)
        : "l"(a), "l"(b), "r"(static_cast<uint32_t>(is)));
}

__device__ __forceinline__ void copy_async(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

// kLanes lanes to a row (16 elements each), 32 / kLanes rows of a token at a time: a pass. A warp's task is
// the passes of a token's queries, then of its keys and its values, or a part of them where tokens are few.
// Rows come through shared memory, three passes ahead (seven: 54 us instead of 45 for 16222 tokens of 28 and
// 4 heads). In registers they took a loop unrolled by four in which no side could follow the other, so
// that a task was one side's, and the few keys' warps had a pass in flight (54 us).
// kAll: all elements of a head are rotated. Where some are not, leaving them alone costs 1 to 2 % on sides with a norm
// (16222 tokens of 64 heads, R 96: 81.7 -> 82.9 us; without one 81.0 -> 80.5) and as much in the cache's kernel
// (576 x 1 to 32 tokens of 32/8 heads, R 64, no norm: 43.7 -> 44.2).
template <bool kF16, int kLanes, bool kPaged, bool kAll>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotateArgs a) {
    __shared__ float2 turned[kWarps][kMaxDim / 2];
    __shared__ uint4 ring[kWarps][kAhead][64];  // the rows of a pass one after another
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kAt = 32 / kLanes;
    const int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
    pdl_wait();
    pdl_launch_next();
    if (task >= a.tasks) return;
    const int64_t x = divide(task, a.chunks);
    const int p_lo = static_cast<int>(task - x * a.chunks) * a.passes, p_hi = min(p_lo + a.passes, a.passes_all);
    const int64_t s = divide(x, a.n_tok);
    const int i = static_cast<int>(x - s * a.n_tok);
    int token = i;
    if (kPaged) {
        int len = a.len[s];
        const int count = a.count ? min(max(a.count[s], 0), a.n_tok) : a.n_tok;
        if (len < 0 || i >= count) return;
        if (len > 0 && (len - 1) >> a.page_log >= a.width) {
            if (lane == 0) flag_error(a.err, RPS_DEVERR_PAGE);
            len = a.width << a.page_log;
        }
        token = len - count + i;
        if (token < 0) return;  // (a row without a place)
    }
    // this lane's 16-byte units of a row
    const int l = lane % kLanes, of_pass = lane / kLanes;
    const bool rotates = l < a.R / 16, there = l < a.D / 16;
    const bool halves = rotates && !a.interleaved;
    const int u0 = (halves ? l : 2 * l) * 16, u1 = (halves ? l + a.R / 16 : 2 * l + 1) * 16;

    // The side of a pass, and the pass that the side begins with.
    const auto side_of = [&](int p, int &begin) -> const Side & {
        if (p < a.passes_q) {
            begin = 0;
            return a.q;
        }
        if (!kPaged || p < a.passes_q + a.passes_k) {
            begin = a.passes_q;
            return a.k;
        }
        begin = a.passes_q + a.passes_k;
        return a.v;
    };
    constexpr uint32_t kSlot = sizeof ring[0][0];
    const uint32_t slots = saddr(&ring[warp][0][0]) + of_pass * 2 * a.D;
    // The units that this lane copies: its own, or (interleaved) side by side with its neighbours', for its
    // own would be fetched by half sectors (16222 tokens of 64 heads: 115 us)
    const int near = a.interleaved ? l * 16 : u0, far = a.interleaved ? near + a.D : u1;
    int begin;
    const Side *in = &side_of(p_lo, begin);
    const char *from = in->src + s * in->src_seq + i * in->src_token + ((p_lo - begin) * kAt + of_pass) * in->src_head;
    int row = (p_lo - begin) * kAt + of_pass;  // of the next pass to be copied
    const auto copy = [&](int p) {
        if (p < p_hi) {
            if (p != p_lo && (p == a.passes_q || (kPaged && p == a.passes_q + a.passes_k))) {  // another side begins
                in = &side_of(p, begin);
                row = of_pass;
                from = in->src + s * in->src_seq + i * in->src_token + row * in->src_head;
            }
            if (there && row < in->heads) {
                const uint32_t to = slots + p % kAhead * kSlot;
                copy_async(to + near, from + near);
                copy_async(to + far, from + far);
            }
            row += kAt;
            from += kAt * in->src_head;
        }
        copies_commit();
    };
#pragma unroll 1
    for (int p = p_lo; p < p_lo + kAhead - 1; ++p) copy(p);

    // the token's place, and its sines and cosines while the rows are on their way
    int64_t place = -1;
    if (kPaged && p_hi > a.passes_q) {
        const int page = a.table[s * a.width + (token >> a.page_log)];
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.n_pages)) {
            if (lane == 0) flag_error(a.err, RPS_DEVERR_PAGE);
        } else if (a.ref[page] > 1) {  // others read this page too
            if (lane == 0) flag_error(a.err, RPS_DEVERR_SHARED);
        } else {
            place = page * a.page_stride + (token & ((1 << a.page_log) - 1)) * a.token_stride;
        }
    }
    if (a.R && p_lo < a.passes_q + a.passes_k) {
        const int64_t t = a.pos ? a.pos[x] : token;
        for (int p = lane; p < a.R / 2; p += 32) {
            const int32_t turn = static_cast<int32_t>(static_cast<uint64_t>(t) * a.turns[p] >> 32);
            float sn, cs;
            sincospif(static_cast<float>(turn) * 0x1p-31f, &sn, &cs);
            turned[warp][p] = make_float2(cs * a.amplitude, sn * a.amplitude);
        }
        __syncwarp();
    }
    const f2 one = pack2(1.f, 1.f), minus = pack2(-1.f, -1.f);
    f2 c0[4], c1[4], s0[4], s1[4];  // w0 cos, w1 cos, w0 sin, -w1 sin
    const Side *d = nullptr;
    char *to = nullptr;
    int at = 0;
    int64_t step = 0;
    bool normed = false, as_is = false, stored = false;
#pragma unroll 1
    for (int p = p_lo; p < p_hi; ++p) {
        if (a.interleaved) __syncwarp();  // (all lanes have taken the pass before, whose place is free)
        copy(p + kAhead - 1);
        if (p == p_lo || p == a.passes_q || (kPaged && p == a.passes_q + a.passes_k)) {  // another side begins
            int first;
            d = &side_of(p, first);
            const bool to_cache = kPaged && p >= a.passes_q;
            normed = d->weight != nullptr;
            // values, and what has neither norm nor rotation, without arithmetic (all lanes alike on a normed side)
            as_is = kPaged && (p >= a.passes_q + a.passes_k || (!kAll && !normed && !rotates));
            at = (p - first) * kAt + of_pass;
            stored = there && (!to_cache || place >= 0);
            const int64_t head = to_cache ? a.head_stride : d->dst_head;
            to = d->dst + at * head + (to_cache ? place : s * d->dst_seq + i * d->dst_token);
            step = kAt * head;
            if (!as_is) {
                f2 w0[4] = {one, one, one, one}, w1[4] = {one, one, one, one};
                if (normed && there)
                    widen16<kF16>(*reinterpret_cast<const uint4 *>(static_cast<const char *>(d->weight) + u0),
                                  *reinterpret_cast<const uint4 *>(static_cast<const char *>(d->weight) + u1), !halves, w0, w1);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float4 f = rotates ? *reinterpret_cast<const float4 *>(&turned[warp][8 * l + 2 * j]) : make_float4(1.f, 0.f, 1.f, 0.f);
                    const f2 cs = pack2(f.x, f.z), sn = pack2(f.y, f.w);
                    c0[j] = mul2(w0[j], cs);
                    c1[j] = mul2(w1[j], cs);
                    s0[j] = mul2(w0[j], sn);
                    s1[j] = mul2(mul2(w1[j], sn), minus);
                }
            }
        }
        copies_wait<kAhead - 1>();
        if (a.interleaved) __syncwarp();
        const uint32_t slot = slots + p % kAhead * kSlot;
        uint4 raw0 = ld_shared_v4(slot + u0), raw1 = ld_shared_v4(slot + u1);
        if (!as_is) {
            f2 y0[4], y1[4];
            widen16<kF16>(raw0, raw1, !halves, y0, y1);
            float r = 1.f;
            if (normed) {
                f2 sum = pack2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum = fma2(y1[j], y1[j], fma2(y0[j], y0[j], sum));
                float lo, hi;
                unpack2(sum, lo, hi);
                lo = there ? lo + hi : 0.f;
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) lo += __shfl_xor_sync(kFull, lo, o);
                r = rsqrtf(lo * a.inv_d + a.eps);
            }
            const f2 rr = pack2(r, r);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f2 z0, z1;
                if (kAll) {
                    z0 = fma2(s1[j], y1[j], mul2(c0[j], y0[j])), z1 = fma2(s0[j], y0[j], mul2(c1[j], y1[j]));
                } else {
                    z0 = mul2(c0[j], y0[j]);
                    fma2_if(z0, s1[j], y1[j], rotates);
                    z1 = mul2(c1[j], y1[j]);
                    fma2_if(z1, s0[j], y0[j], rotates);
                }
                if (normed) {
                    z0 = mul2(z0, rr);
                    z1 = mul2(z1, rr);
                }
                y0[j] = z0;
                y1[j] = z1;
            }
            narrow16<kF16>(y0, y1, !halves, raw0, raw1);
        }
        // (from tensor to tensor such lanes go along and take their elements again: a jump around the arithmetic took
        // 83.9 us instead of 82.9 for the 16222 tokens above; in the cache's kernel this took 50.2 instead of 44.2)
        if (!kPaged && !kAll && !normed && !rotates) {
            raw0 = ld_shared_v4(slot + u0);
            raw1 = ld_shared_v4(slot + u1);
        }
        if (stored && at < d->heads) {
            *reinterpret_cast<uint4 *>(to + u0) = raw0;
            *reinterpret_cast<uint4 *>(to + u1) = raw1;
        }
        at += kAt;
        to += step;
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
    const auto passes = [&](int heads) { return (heads + at - 1) / at; };
    a.passes_q = passes(a.q.heads);
    a.passes_k = passes(a.k.heads);
    a.passes_all = a.passes_q + a.passes_k + (kPaged ? passes(a.v.heads) : 0);
    // Tokens are split where there are too few: down to single passes until the card is full, for they come one
    // after another, and to eight, which carry a token's sines and cosines, until there are eight tasks for each
    // warp, so that the last ones of the call are short.
    const int64_t warps = static_cast<int64_t>(sms) * kFullWarps;
    const int64_t fill = std::min<int64_t>(a.passes_all, warps / tokens), even = std::min<int64_t>(a.passes_all / 8, 8 * warps / tokens);
    a.chunks = static_cast<int32_t>(std::max<int64_t>({1, fill, even}));
    a.passes = (a.passes_all + a.chunks - 1) / a.chunks;
    a.chunks = (a.passes_all + a.passes - 1) / a.passes;
    a.tasks = tokens * a.chunks;
    const int64_t blocks = (a.tasks + kWarps - 1) / kWarps;
    if (blocks > INT32_MAX) return RPS_ERR_UNSUPPORTED;
    const auto pick = [&](auto all) {
        constexpr bool kAll = decltype(all)::value;
        return lanes == 4   ? (f16 ? rotate_kernel<true, 4, kPaged, kAll> : rotate_kernel<false, 4, kPaged, kAll>)
               : lanes == 8 ? (f16 ? rotate_kernel<true, 8, kPaged, kAll> : rotate_kernel<false, 8, kPaged, kAll>)
                            : (f16 ? rotate_kernel<true, 16, kPaged, kAll> : rotate_kernel<false, 16, kPaged, kAll>);
    };
    const auto kernel = a.R == a.D ? pick(std::true_type{}) : pick(std::false_type{});
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
