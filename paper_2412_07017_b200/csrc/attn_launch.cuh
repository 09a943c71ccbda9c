// Host side that the attention kernels' launchers share: tensor maps of the pools, the shared-memory attribute, the
// warp body's stages.
#pragma once
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "attn_decode.cuh"
#include "kernels.h"

namespace asynclm {

namespace {

constexpr int kMaxSmem = 232448;

__device__ __forceinline__ uint8_t* aligned_smem(uint8_t* raw) {
    return (uint8_t*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

typedef CUresult (*ReplaceAddressFn)(CUtensorMap*, void*);

// The pool as the two bodies read it, landed with the 128-byte swizzle:
//   kv    (64 values, 16 slots, d / 64 row halves, Hkv, pages x K|V), a box is one page's K and V blocks of one kv head
//         (dec::tma_page_kv)
//   span  (64 values, 8 slots, d / 64 row halves, 2 groups of 8 slots, pages x K|V x Hkv), a box is one block
// (tc::tma_page)
//   kv8   the 8-bit cache: (d bytes, 16 slots, Hkv, pages x K|V), a box as kv's; at head_dim 64 with the 64-byte
// swizzle (dec::tma_page_kv8)
//   k8    the same, a box is one block (tc::kv8_k_producer)
enum PoolMap { kKvMap, kSpanMap, kKv8Map, kK8Map };

constexpr int64_t kMaxMapPages = 0x3fffffff;

cudaError_t make_pool_map(PoolMap kind, const DevPlan& p, const void* pool, CUtensorMap* map) {
    static std::atomic<EncodeTiledFn> encode_fn{nullptr};
    EncodeTiledFn encode = encode_fn.load(std::memory_order_acquire);
    if (encode == nullptr) {
        cudaError_t e = driver_function("cuTensorMapEncodeTiled", &encode);
        if (e != cudaSuccess) return e;
        encode_fn.store(encode, std::memory_order_release);
    }
    const cuuint64_t d = (cuuint64_t)p.head_dim, hkv = (cuuint64_t)p.num_kv_heads;
    if (p.num_pages <= 0) return cudaErrorInvalidValue;
    // (the pages that a tensor map can count hold more than any device's memory)
    const cuuint64_t blocks = 2 * (cuuint64_t)std::min(p.num_pages, kMaxMapPages);
    const cuuint64_t dims_kv[5] = {64, kPage, d / 64, hkv, blocks}, strides_kv[4] = {d * 2, 128, kPage * d * 2, hkv * kPage * d * 2};
    const cuuint64_t dims_span[5] = {64, 8, d / 64, 2, std::min<cuuint64_t>(blocks * hkv, INT32_MAX)};
    const cuuint64_t strides_span[4] = {d * 2, 128, 8 * d * 2, kPage * d * 2};
    const cuuint32_t box_kv[5] = {64, kPage, (cuuint32_t)(d / 64), 1, 2}, box_span[5] = {64, 8, (cuuint32_t)(d / 64), 2, 1};
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    if (kind == kKv8Map || kind == kK8Map) {
        const cuuint64_t dims[4] = {d, kPage, hkv, blocks}, strides[3] = {d, kPage * d, hkv * kPage * d};
        const cuuint32_t box[4] = {(cuuint32_t)d, kPage, 1, kind == kKv8Map ? 2u : 1u};
        const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(pool), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                  d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
    }
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(pool), kind == kKvMap ? dims_kv : dims_span,
                              kind == kKvMap ? strides_kv : strides_span, kind == kKvMap ? box_kv : box_span, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// cudaFuncSetAttribute(MaxDynamicSharedMemorySize) once per kernel and device instead of once per launch.
// The kernel is a template VALUE: kernels of one signature share a pointer type, and a flag per type
// would let the first of them stand for all.
template <auto kernel>
cudaError_t allow_smem(size_t bytes) {
    static std::atomic<unsigned long long> done{0};      // one per kernel instantiation; bit = device (first 64)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
    if (bit != 0 && (done.load(std::memory_order_acquire) & bit) != 0) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess && bit != 0) done.fetch_or(bit, std::memory_order_release);
    return e;
}

// A pool's tensor map: that of its shape, of which the last few are kept per thread and kind, with its address put in.
// (The layers of a model have a pool each; encoding a launch's map anew takes longer than the address.)
cudaError_t pool_map(PoolMap kind, const DevPlan& p, const void* pool, CUtensorMap* map) {
    struct Entry { int64_t pages; int hkv, d; CUtensorMap map; };
    constexpr int kEntries = 8;
    thread_local Entry cache[4][kEntries] = {};
    thread_local int next[4] = {};
    static std::atomic<ReplaceAddressFn> replace_fn{nullptr};
    ReplaceAddressFn replace = replace_fn.load(std::memory_order_acquire);
    if (replace == nullptr) {
        cudaError_t e = driver_function("cuTensorMapReplaceAddress", &replace);
        if (e != cudaSuccess) return e;
        replace_fn.store(replace, std::memory_order_release);
    }
    for (const Entry& x : cache[kind])
        if (x.pages == p.num_pages && x.hkv == p.num_kv_heads && x.d == p.head_dim) {
            *map = x.map;
            return replace(map, const_cast<void*>(pool)) == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
        }
    const cudaError_t e = make_pool_map(kind, p, pool, map);
    if (e == cudaSuccess) {
        cache[kind][next[kind]] = Entry{p.num_pages, p.num_kv_heads, p.head_dim, *map};
        next[kind] = (next[kind] + 1) % kEntries;
    }
    return e;
}

template <int D, bool KV8 = false>
constexpr int decode_stages() {
    int S = dec::kMaxStages;
    while (S > 2 && dec::smem_bytes<D, KV8>(S) > (size_t)kMaxSmem) --S;
    return S;
}

}  // namespace

}  // namespace asynclm
