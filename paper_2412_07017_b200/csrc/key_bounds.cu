// Least and largest value of every key channel of a page: what a page's score is taken from (select_pages.cu).
//
// A warp takes one (page, kv head): 16 slots of head_dim values, read as 16-byte vectors (a row is 16 or 8 lanes of bf16, 8 or 4 of 8-bit
// codes), folded per lane, then over the lanes that hold the same channels.  Bound by the bytes of K: one pass, nothing is kept between
// calls, so a page that is appended to is read again as a whole (16 rows of one page a kv head for a decoding sequence).  All of 164 K tokens, 8 kv heads of
// 128: 62.6 us, 6.07 TB/s, 0.94 of a copy's rate; 48 sequences' pages of one to four new tokens 1.9 us.  Of the 8-bit cache 75 us (32.8 at the copy's rate) and 2.7: there a
// pair of codes takes a decoding, two products and a packing that the 16-bit form has not; what of it bounds has not been separated.
#include <algorithm>

#include "asynclm.h"
#include "kernels.h"
#include "kv8.cuh"
#include "plan_internal.h"

namespace asynclm {

namespace {

constexpr int kBoundWarps = 8;

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The pair with NaN replaced by `inf` (a channel that holds one is bounded by nothing).
__device__ __forceinline__ uint32_t no_nan(uint32_t w, uint32_t inf) {
    if ((w & 0x7fffu) > 0x7f80u) w = (w & 0xffff0000u) | inf;
    if ((w >> 16 & 0x7fffu) > 0x7f80u) w = (w & 0xffffu) | inf << 16;
    return w;
}

// FROM_START: an entry is one of the page table, else a new row, and its page is that of the first new row in it.
template <int D, bool KV8, bool FROM_START>
__global__ void __launch_bounds__(32 * kBoundWarps)
key_bounds_kernel(DevPlan p, const uint8_t* __restrict__ pool, const uint8_t* __restrict__ scales, uint8_t* __restrict__ bounds) {
    constexpr int kLanes = D * (KV8 ? 1 : 2) / 16;           // of a row
    constexpr int kRows = 32 / kLanes, kLoads = kPage / kRows;
    constexpr int kPairs = KV8 ? 8 : 4;                       // of a lane's vector
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * kBoundWarps + (threadIdx.x >> 5);
    const int64_t entry = w / p.num_kv_heads;
    const int h = (int)(w % p.num_kv_heads);
    int64_t page = -1;
    int used = 0;
    if (FROM_START) {
        if (entry < p.total_pages) {
            int lo = 0, hi = p.batch;      // the last sequence whose pages start at or before the entry
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (__ldg(p.page_indptr + mid) <= entry) lo = mid; else hi = mid;
            }
            const int new_rows = __ldg(p.q_indptr + lo + 1) - __ldg(p.q_indptr + lo);
            const int64_t end = (int64_t)__ldg(p.kv_len_before + lo) + new_rows, at = (entry - __ldg(p.page_indptr + lo)) * kPage;
            if (new_rows > 0 && at < end) {
                used = (int)min((int64_t)kPage, end - at);
                page = __ldg(p.page_indices + entry);
            }
        }
    } else if (entry < p.total_q) {
        const int r = (int)entry, seq = __ldg(p.row_seq + r), r0 = __ldg(p.q_indptr + seq), r1 = __ldg(p.q_indptr + seq + 1);
        const int64_t at = __ldg(p.row_slot + r);
        const int slot = (int)(at % kPage);
        if (slot == 0 || r == r0) {
            used = min(kPage, slot + r1 - r);
            page = at / kPage;
        }
    }
    pdl_wait();      // the pool belongs to the kernels in front until they have completed
    if (used == 0 || !page_ok(page, p.num_pages, p.status, kStatusBadPageBounds)) return;
    const int row0 = lane / kLanes, piece = lane % kLanes;
    uint32_t lo[kPairs], hi[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) lo[i] = 0x7f807f80u, hi[i] = 0xff80ff80u;
    const uint8_t* src = pool + pool_row_offset(page, 0, h, 0, p.num_kv_heads, D) * (KV8 ? 1 : 2) + (size_t)lane * 16;
    uint4 v[kLoads];
    uint32_t e[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int slot = i * kRows + row0;
        if (slot < used) {
            v[i] = *reinterpret_cast<const uint4*>(src + (size_t)i * kRows * kLanes * 16);
            if (KV8) e[i] = scales[kv8_scale_offset(page, 0, h, slot, p.num_kv_heads)];
        }
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        if (i * kRows + row0 >= used) continue;
        const uint32_t x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
        if constexpr (KV8) {
            const float s = kv8_scale(e[i]);
#pragma unroll
            for (int k = 0; k < kPairs; ++k) {      // (a code times its scale is a bf16 value)
                const uint32_t c = k & 1 ? kv8_decode2_hi(x[k / 2]) : kv8_decode2(x[k / 2]);
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&c));
                const uint32_t b = pack_bf16x2(f.x * s, f.y * s);
                lo[k] = min2(lo[k], b);
                hi[k] = max2(hi[k], b);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kPairs; ++k) {
                lo[k] = min2(lo[k], x[k]);
                hi[k] = max2(hi[k], x[k]);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
#pragma unroll
        for (int off = kLanes; off < 32; off <<= 1) {
            lo[k] = min2(lo[k], __shfl_xor_sync(0xffffffffu, lo[k], off));
            hi[k] = max2(hi[k], __shfl_xor_sync(0xffffffffu, hi[k], off));
        }
        lo[k] = no_nan(lo[k], 0xff80u);
        hi[k] = no_nan(hi[k], 0x7f80u);
    }
    if (row0 > 1) return;
    // the first row's lanes write the least values, the second's the largest
    uint4* dst = reinterpret_cast<uint4*>(bounds + (((size_t)page * p.num_kv_heads + h) * 2 + row0) * D * 2) + piece * (kPairs / 4);
#pragma unroll
    for (int k = 0; k < kPairs; k += 4)
        dst[k / 4] = row0 ? make_uint4(hi[k], hi[k + 1], hi[k + 2], hi[k + 3]) : make_uint4(lo[k], lo[k + 1], lo[k + 2], lo[k + 3]);
}

template <int D, bool KV8>
cudaError_t launch_bounds(const DevPlan& p, const void* pool, const void* scales, void* bounds, bool from_start, cudaStream_t s) {
    const int64_t warps = (from_start ? p.total_pages : (int64_t)p.total_q) * p.num_kv_heads, blocks = (warps + kBoundWarps - 1) / kBoundWarps;
    if (blocks == 0) return cudaSuccess;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    return launch_when(!p.full_launch, from_start ? key_bounds_kernel<D, KV8, true> : key_bounds_kernel<D, KV8, false>, dim3((unsigned)blocks),
                      dim3(32 * kBoundWarps), 0, s, p, (const uint8_t*)pool, (const uint8_t*)scales, (uint8_t*)bounds);
}

int key_bounds(const asynclm_plan_t* plan, const void* pool, const void* scales, bool kv8, void* bounds, int32_t from_start, void* stream) {
    if (!plan || plan->magic != kPlanMagic || plan->host_only) return ASYNCLM_ERR_INVALID_ARG;
    if (plan->dev.total_q == 0) return ASYNCLM_OK;
    if (!pool || !bounds || (kv8 && !scales) || (((uintptr_t)pool | (uintptr_t)scales | (uintptr_t)bounds) & 15) != 0) return ASYNCLM_ERR_INVALID_ARG;
    if (int rc = check_plan_device(plan->device)) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    PlanUse use(plan, s);
    const bool wide = use.dev.head_dim == 128;
    const bool all = from_start != 0;
    const cudaError_t e = kv8 ? (wide ? launch_bounds<128, true>(use.dev, pool, scales, bounds, all, s) : launch_bounds<64, true>(use.dev, pool, scales, bounds, all, s))
                              : (wide ? launch_bounds<128, false>(use.dev, pool, nullptr, bounds, all, s) : launch_bounds<64, false>(use.dev, pool, nullptr, bounds, all, s));
    return cuda_status(use.launched(e));
}

}  // namespace

}  // namespace asynclm

extern "C" int asynclm_kv_bounds(const asynclm_plan_t* plan, const void* kv_pool, void* key_bounds, int32_t from_start, void* stream) {
    return asynclm::key_bounds(plan, kv_pool, nullptr, false, key_bounds, from_start, stream);
}

extern "C" int asynclm_kv8_bounds(const asynclm_plan_t* plan, const void* kv8_pool, const void* kv8_scales, void* key_bounds, int32_t from_start, void* stream) {
    return asynclm::key_bounds(plan, kv8_pool, kv8_scales, true, key_bounds, from_start, stream);
}
