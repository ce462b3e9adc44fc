// kv_maps.cuh -- the tensor maps through which the attention kernels copy the pages
// of the K/V cache, and the rows of queries, with TMA.
#pragma once

#include <cuda.h>  // CUtensorMap and the tensor-map encoder's signature (no link against the driver)
#include <cudaTypedefs.h>

#include <mutex>

#include "rps_internal.cuh"

namespace rps {
namespace {

constexpr int kHeadDim = 128;
typedef PFN_cuTensorMapEncodeTiled_v12000 Encoder;

// The driver's encoder (nullptr: not available).
Encoder tensor_map_encoder() {
    static std::mutex mutex;
    static Encoder known = nullptr;
    std::lock_guard<std::mutex> lock(mutex);
    if (!known) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            known = reinterpret_cast<Encoder>(fn);
    }
    return known;
}

// A copy of K or V takes 2^copy_log tokens. by_groups: from a map whose third dimension goes
// through the tokens of all pages by eights, page_groups of them a page; else 8 tokens of a page.
struct PageCopies {
    int32_t by_groups, copy_log, page_groups, no_page;  // no_page: a coordinate beyond the pages
};

// A map of 16-bit elements: extents, strides (in elements) and boxes from the inner dimension
// (64-wide boxes of kHeadDim contiguous elements, or 64) outwards.
template <int n>
rps_status make_map(Encoder encode, CUtensorMap *m, const void *base, bool f16, int64_t inner, const int64_t (&ext)[n],
                    const int64_t (&stride)[n], const uint32_t (&box)[n]) {
    cuuint64_t dims[n + 1] = {static_cast<cuuint64_t>(inner)}, bytes[n];
    cuuint32_t boxes[n + 1] = {64}, es[n + 1] = {1};
    for (int i = 0; i < n; ++i) {
        dims[i + 1] = static_cast<cuuint64_t>(ext[i]);
        // (the stride of a dimension of one is not used, but has to be a valid one)
        bytes[i] = static_cast<cuuint64_t>(ext[i] > 1 ? stride[i] : kHeadDim) * 2;
        boxes[i + 1] = box[i];
        es[i + 1] = 1;
    }
    const CUresult r = encode(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, n + 1,
                                       const_cast<void *>(base), dims, bytes, boxes, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? RPS_OK : RPS_ERR_CUDA;
}

// The maps of K and V: a copy brings whole groups of 8 tokens, both halves of their columns.
// Where the pages' stride is a multiple of eight tokens', one dimension goes through the groups
// of all pages, and a copy takes a slot; else a copy is a group of one page.
// slot_log: of a slot, min(page_size, 128) tokens.
rps_status map_pages(Encoder encode, CUtensorMap *tk, CUtensorMap *tv, const rps_kv_cache *kv, int32_t layer, int slot_log,
                     PageCopies &a) {
    const bool f16 = kv->dtype == RPS_F16;
    const int64_t layer_at = kv->n_layers > 1 ? layer * kv->layer_stride * 2 : 0;
    const int64_t groups = kv->page_size / 8, token = kv->token_stride, group = 8 * token;
    const int64_t per_page = kv->n_pages > 1 ? kv->page_stride / group : groups;
    const int64_t all = (kv->n_pages - 1) * per_page + groups;
    const void *const base[2] = {static_cast<char *>(kv->k) + layer_at, static_cast<char *>(kv->v) + layer_at};
    CUtensorMap *const to[2] = {tk, tv};
    a.by_groups = (kv->n_pages == 1 || kv->page_stride % group == 0) && all <= INT32_MAX;
    a.copy_log = a.by_groups ? slot_log : 3;
    a.page_groups = a.by_groups ? static_cast<int32_t>(per_page) : 0;
    a.no_page = a.by_groups ? static_cast<int32_t>(all) : kv->n_pages;
    for (int i = 0; i < 2; ++i) {
        rps_status st;
        if (a.by_groups) {
            const int64_t ext[4] = {8, 2, all, kv->n_heads}, stride[4] = {token, 64, group, kv->head_stride};
            const uint32_t box[4] = {8, 2, (1u << slot_log) / 8, 1};
            st = make_map(encode, to[i], base[i], f16, 64, ext, stride, box);
        } else {
            const int64_t ext[4] = {kv->page_size, 2, kv->n_heads, kv->n_pages};
            const int64_t stride[4] = {token, 64, kv->head_stride, kv->page_stride};
            const uint32_t box[4] = {8, 2, 1, 1};
            st = make_map(encode, to[i], base[i], f16, 64, ext, stride, box);
        }
        if (st != RPS_OK) return st;
    }
    return RPS_OK;
}

}  // namespace
}  // namespace rps
