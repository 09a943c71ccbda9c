// The 8-bit cache read back: ranges of sequences as dense bf16 rows.
//
// Output row out_indptr[b] + i is position first[b] + i of sequence b, found through the plan's page table; its values
// are code * 2^e, exact in bf16.  Bound by memory: d + 1 bytes read and 2 d written for each K or V row.  A thread
// turns 8 codes into 16 bytes; head_dim / 8 lanes take a row, a warp 2 or 4 rows that follow each other, which in the
// pool are next to each other inside a page (and in the output Hkv rows apart, whole 128-byte lines each). (With 16
// codes to a thread every store instruction leaves half of each 32-byte sector to the next one.)  The row's place is
// looked up once, by bisection over out_indptr, and serves all its heads.  133 K tokens of 8 heads of 128 take 129-136
// us, 6.0-6.3 TB/s; 700 of 2 heads of 64 2.4 in a graph.
#include <algorithm>

#include "kernels.h"
#include "kv8.cuh"
#include "plan_internal.h"

namespace asynclm {

namespace {

constexpr int kGatherThreads = 256;
constexpr int kGatherUnroll = 8;

__global__ void __launch_bounds__(kGatherThreads)
kv8_gather_kernel(DevPlan p, const int64_t* out_indptr, const int32_t* first, const uint8_t* __restrict__ pool, const uint8_t* __restrict__ scales,
                  uint4* __restrict__ k_out, uint4* __restrict__ v_out, int64_t total, int heads_per_cta) {
    pdl_trigger();
    pdl_wait();
    const int d = p.head_dim, hkv = p.num_kv_heads, per_row = d / 8;
    const int v = threadIdx.x % per_row;
    const int64_t row = (int64_t)blockIdx.x * (kGatherThreads / per_row) + threadIdx.x / per_row;
    if (row >= total) return;
    // the sequence: the last b with out_indptr[b] <= row (empty ranges are passed over)
    int lo = 0, hi = p.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(out_indptr + mid) <= row) lo = mid; else hi = mid;
    }
    const int b = lo;
    const int64_t i = row - __ldg(out_indptr + b), pos = __ldg(first + b) + i;
    const int64_t length = (int64_t)__ldg(p.kv_len_before + b) + __ldg(p.q_indptr + b + 1) - __ldg(p.q_indptr + b);
    const int64_t at = (int64_t)__ldg(p.page_indptr + b) + pos / kPage;
    // Ranges come from device memory and the planner does not look at the pages of sequences without new tokens:
    // whatever lies outside the sequence, its pages or the pool is reported and left out.
    int64_t page = -1;
    if (i >= 0 && row < __ldg(out_indptr + b + 1) && pos >= 0 && pos < length && at < __ldg(p.page_indptr + b + 1)) page = __ldg(p.page_indices + at);
    if (page < 0 || page >= p.num_pages) {
        atomicCAS(p.status, 0, kStatusBadGather);
        return;
    }
    const int slot = (int)(pos % kPage);
    const int c0 = blockIdx.y * heads_per_cta, c1 = min(c0 + heads_per_cta, 2 * hkv);      // (kv head, K|V) pairs, K heads first
    for (int c = c0; c < c1; c += kGatherUnroll) {
        uint2 codes[kGatherUnroll];
        uint32_t byte[kGatherUnroll];
#pragma unroll
        for (int u = 0; u < kGatherUnroll; ++u) {
            const int which = c + u >= hkv, h = c + u - which * hkv;
            if (c + u < c1) {
                codes[u] = __ldcg(reinterpret_cast<const uint2*>(pool + kv8_row_offset(page, which, h, slot, hkv, d) + 8 * v));
                byte[u] = __ldcg(scales + kv8_scale_offset(page, which, h, slot, hkv));
            }
        }
#pragma unroll
        for (int u = 0; u < kGatherUnroll; ++u) {
            if (c + u >= c1) break;
            const int which = c + u >= hkv, h = c + u - which * hkv;
            const float s = kv8_scale(byte[u]);
            const uint32_t w[2] = {codes[u].x, codes[u].y};
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t a = kv8_decode2(w[k]), bb = kv8_decode2_hi(w[k]);
                const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&a)), fb = __half22float2(*reinterpret_cast<const __half2*>(&bb));
                o[2 * k] = pack_bf16x2(fa.x * s, fa.y * s);
                o[2 * k + 1] = pack_bf16x2(fb.x * s, fb.y * s);
            }
            (which ? v_out : k_out)[((size_t)row * hkv + h) * (d / 8) + v] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

}  // namespace

}  // namespace asynclm

extern "C" int asynclm_kv8_gather(const asynclm_plan_t* plan, const int64_t* out_indptr, const int32_t* first, int64_t total_rows, const void* kv8_pool,
                                  const void* kv8_scales, void* k_out, void* v_out, void* stream) {
    using namespace asynclm;
    if (!plan || plan->magic != kPlanMagic || plan->host_only || total_rows < 0) return ASYNCLM_ERR_INVALID_ARG;
    if (total_rows == 0) return ASYNCLM_OK;
    const DevPlan& d = plan->dev;
    if (d.batch == 0 || !out_indptr || !first || !kv8_pool || !kv8_scales || !k_out || !v_out || ((uintptr_t)out_indptr & 7) != 0 || ((uintptr_t)first & 3) != 0 ||
        (((uintptr_t)kv8_pool | (uintptr_t)kv8_scales | (uintptr_t)k_out | (uintptr_t)v_out) & 15) != 0)
        return ASYNCLM_ERR_INVALID_ARG;
    if (int rc = check_plan_device(plan->device)) return rc;
    const int rows = kGatherThreads / (d.head_dim / 8);
    const int64_t ctas = (total_rows + rows - 1) / rows;
    if (ctas > INT32_MAX) return ASYNCLM_ERR_INVALID_ARG;
    // few rows: their heads are spread over more CTAs, until the SMs have a few each
    int per_cta = 2 * d.num_kv_heads;
    while (per_cta > kGatherUnroll && ctas * ((2 * d.num_kv_heads + per_cta - 1) / per_cta) < 148 * 4) per_cta = (per_cta + 1) / 2;
    PlanUse use(plan, (cudaStream_t)stream);
    return cuda_status(use.launched(launch_when(!use.dev.full_launch, kv8_gather_kernel, dim3((unsigned)ctas, (2 * d.num_kv_heads + per_cta - 1) / per_cta),
                                                dim3(kGatherThreads), 0, (cudaStream_t)stream, use.dev, out_indptr, first, (const uint8_t*)kv8_pool,
                                                (const uint8_t*)kv8_scales, (uint4*)k_out, (uint4*)v_out, total_rows, per_cta)));
}
