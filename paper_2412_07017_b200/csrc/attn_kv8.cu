// Attention over the 8-bit cache: the entry point, its kernels and launcher.  The bodies are those of the bf16 cache,
// with the cache's format as a template parameter (attn_decode.cuh: what a consumer warp does with a page;
// attn_append_tc.cuh: how tiles get into shared memory).  Which kernel runs follows the same rules as there
// (attn_kernels.cu).
//
// Decode is bound by memory, at half the bytes: 64 sequences of 1-3 K keys, 32 / 8 heads of 128, 51-53 us (4.9-5 TB/s),
// 5 of 32-110 K 145-154 (5.5-5.8 TB/s).
// Spans are bound by the softmax warps' chain: 64 keys take a CTA alone, at head_dim 128, 0.85 us with one row tile and
// 1.35 with two (0.46 | 0.81 in 16 bits), with all SMs at work 1.16 | 1.37 (0.73 | 1.19).  Without the conversion of V
// 0.82 | 1.26 alone, without the reading of the keys' scales (64 values to each of eight warps, from shared memory)
// 0.81 | 1.20: neither is the bound by itself. 8 spans of 8-64 tokens beside 24 decode rows over 0.5-4 K keys 75-81 us
// (a batch of the same kind in 16 bits 64; without either of the two, other such batches take 0.95 to 1 of their time),
// a prompt of 7777 tokens 684-707 us, 701-724 TFLOP/s.  The kernel of both bodies spills: an 88-byte frame at four
// heads of 128, because its registers are split once for both.
#include "asynclm.h"
#include "attn_append_tc.cuh"
#include "attn_decode.cuh"
#include "attn_launch.cuh"
#include "plan_internal.h"

namespace asynclm {

namespace {

template <int D, int G>
__global__ void __launch_bounds__(dec::kThreads, 1)
attn_decode_kv8_kernel(DevPlan p, const __grid_constant__ CUtensorMap kv_map, const uint8_t* pool, const uint8_t* scales, const __nv_bfloat16* __restrict__ q,
                       __nv_bfloat16* __restrict__ out, float* __restrict__ lse, int S) {
    extern __shared__ uint8_t smem_raw[];
    pdl_trigger();      // the kernel behind this one may start its prologue
    if (threadIdx.x == 0) { trace_mark(0); trace_set(1, 0); trace_set(5, 0); trace_set(6, 0); trace_set(7, 0); }
    dec::decode_body<D, G, false, true, true>(p, &kv_map, reinterpret_cast<const __nv_bfloat16*>(pool), q, out, lse, S, aligned_smem(smem_raw), AppendSrc{}, scales);
}

template <int D, int G, int ROLE>
__device__ __forceinline__ void span_kv8(const DevPlan& p, const CUtensorMap* k_map, const uint8_t* pool, const uint8_t* scales, const __nv_bfloat16* __restrict__ q,
                                         __nv_bfloat16* __restrict__ out, float* __restrict__ lse, uint8_t* smem) {
    tc::split_registers<ROLE>();
    tc::tc_body<D, G, true, true, ROLE>(p, k_map, q, nullptr, out, lse, smem, pool, scales);
}

template <int D, int G>
__global__ void __launch_bounds__(tc::kThreadsKv8, 1)
attn_append_tc_kv8_kernel(DevPlan p, const __grid_constant__ CUtensorMap k_map, const uint8_t* pool, const uint8_t* scales, const __nv_bfloat16* __restrict__ q, __nv_bfloat16* __restrict__ out,
                          float* __restrict__ lse) {
    extern __shared__ uint8_t smem_raw[];
    pdl_trigger();
    if (threadIdx.x == 0) {
        trace_mark(0);
        for (int s = 8; s < 16; ++s) trace_set(s, 0);
    }
    if (threadIdx.x < 256) span_kv8<D, G, 0>(p, &k_map, pool, scales, q, out, lse, aligned_smem(smem_raw));
    else span_kv8<D, G, 1>(p, &k_map, pool, scales, q, out, lse, aligned_smem(smem_raw));
    if (threadIdx.x == 0) trace_mark(1);
}

template <int D, int G, int ROLE>
__device__ __forceinline__ void fused_kv8(const DevPlan& p, const CUtensorMap* kv_map, const CUtensorMap* k_map, const uint8_t* pool, const uint8_t* scales,
                                          const __nv_bfloat16* __restrict__ q, __nv_bfloat16* __restrict__ out, float* __restrict__ lse, int S, uint8_t* smem) {
    tc::split_registers<ROLE>();
    const int32_t* head = p.cta_heads + (size_t)blockIdx.x * kHeadWords;
    if (head[0] != head[1]) {
        if (threadIdx.x == 0) {
            for (int s = 8; s < 16; ++s) trace_set(s, 0);
        }
        tc::tc_body<D, G, false, true, ROLE>(p, k_map, q, nullptr, out, lse, smem, pool, scales);
        if (threadIdx.x == 0) trace_mark(1);
        if (head[2] == head[3] && p.queue_count == 0) return;      // nothing left for the warp body
        // (as in attn_fused_kernel)
        if (head[2] == head[3] && p.num_join_blocks > 0) {
            if (!dec::queue_has_items(p)) return;
        } else {
            __syncthreads();
        }
    }
    dec::decode_body<D, G, false, false, true, ROLE>(p, kv_map, nullptr, q, out, lse, S, smem, AppendSrc{}, scales);
}

template <int D, int G>
__global__ void __launch_bounds__(tc::kThreadsKv8, 1)
attn_fused_kv8_kernel(DevPlan p, const __grid_constant__ CUtensorMap kv_map, const __grid_constant__ CUtensorMap k_map, const uint8_t* pool, const uint8_t* scales, const __nv_bfloat16* __restrict__ q,
                      __nv_bfloat16* __restrict__ out, float* __restrict__ lse, int S) {
    extern __shared__ uint8_t smem_raw[];
    pdl_trigger();
    if (threadIdx.x == 0) { trace_mark(0); trace_set(1, 0); trace_set(5, 0); trace_set(6, 0); trace_set(7, 0); }
    const int32_t* head = p.cta_heads + (size_t)blockIdx.x * kHeadWords;
    if (threadIdx.x < 3) asm volatile("prefetch.global.L2 [%0];" ::"l"(head + 32 * threadIdx.x));      // (as in attn_fused_kernel)
    if (threadIdx.x == 32) asm volatile("prefetch.tensormap [%0];" ::"l"(&kv_map));
    if (threadIdx.x < 256) fused_kv8<D, G, 0>(p, &kv_map, &k_map, pool, scales, q, out, lse, S, aligned_smem(smem_raw));
    else fused_kv8<D, G, 1>(p, &kv_map, &k_map, pool, scales, q, out, lse, S, aligned_smem(smem_raw));
}

template <int D, int G>
cudaError_t launch_kv8_impl(const DevPlan& p, const void* q, const void* pool, const void* scales, void* out, float* lse, cudaStream_t stream) {
    const bool has_tensor = p.num_items_tensor > 0, has_cuda = p.num_items_cuda > 0;
    if (!has_tensor && !has_cuda) return cudaSuccess;
    if (p.num_pages > kMaxMapPages) return cudaErrorInvalidValue;
    constexpr int S = decode_stages<D, true>();
    constexpr size_t smem_warp = dec::smem_bytes<D, true>(S), smem_span = tc::Geometry<D, true>::SMEM_BYTES, smem_both = std::max(smem_warp, smem_span);
    static_assert(S == dec::Geometry<D, true>::KV8_STAGES, "as many stages as fit");
    static_assert(smem_warp - 1024 <= tc::Geometry<D, true>::OFF_BAR, "the span body's barriers stay clear of the warp body");
    const auto *pool8 = (const uint8_t*)pool, *scales8 = (const uint8_t*)scales;
    const auto* q16 = (const __nv_bfloat16*)q;
    auto* out16 = (__nv_bfloat16*)out;
    CUtensorMap map, k_map;
    if (has_cuda)
        if (cudaError_t e = pool_map(kKv8Map, p, pool, &map)) return e;
    if (has_tensor)
        if (cudaError_t e = pool_map(kK8Map, p, pool, &k_map)) return e;
    if (has_tensor && has_cuda && p.num_ctas_tensor == p.num_ctas_cuda) {
        if (cudaError_t e = allow_smem<attn_fused_kv8_kernel<D, G>>(smem_both)) return e;
        return launch_when(!p.full_launch, attn_fused_kv8_kernel<D, G>, dim3(p.num_ctas_cuda), dim3(tc::kThreadsKv8), smem_both, stream, p, map, k_map, pool8, scales8,
                           q16, out16, lse, S);
    }
    if (has_tensor) {
        if (cudaError_t e = allow_smem<attn_append_tc_kv8_kernel<D, G>>(smem_span)) return e;
        if (cudaError_t e = launch_when(!p.full_launch, attn_append_tc_kv8_kernel<D, G>, dim3(p.num_ctas_tensor), dim3(tc::kThreadsKv8), smem_span, stream, p, k_map,
                                        pool8, scales8, q16, out16, lse))
            return e;
    }
    if (!has_cuda) return cudaSuccess;
    if (cudaError_t e = allow_smem<attn_decode_kv8_kernel<D, G>>(smem_warp)) return e;
    return launch_when(!p.full_launch, attn_decode_kv8_kernel<D, G>, dim3(p.num_ctas_cuda), dim3(dec::kThreads), smem_warp, stream, p, map, pool8, scales8, q16,
                       out16, lse, S);
}

template <int D>
cudaError_t launch_kv8_d(const DevPlan& p, const void* q, const void* pool, const void* scales, void* out, float* lse, cudaStream_t stream) {
    switch (p.group) {
        case 1: return launch_kv8_impl<D, 1>(p, q, pool, scales, out, lse, stream);
        case 2: return launch_kv8_impl<D, 2>(p, q, pool, scales, out, lse, stream);
        case 4: return launch_kv8_impl<D, 4>(p, q, pool, scales, out, lse, stream);
        case 8: return launch_kv8_impl<D, 8>(p, q, pool, scales, out, lse, stream);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace

}  // namespace asynclm

extern "C" int asynclm_kv8_attn_mixed(const asynclm_plan_t* plan, const void* q, const void* kv8_pool, const void* kv8_scales, void* out, float* lse,
                                      void* stream) {
    using namespace asynclm;
    if (!plan || plan->magic != kPlanMagic || plan->host_only) return ASYNCLM_ERR_INVALID_ARG;
    if (plan->dev.total_q == 0) return ASYNCLM_OK;
    if (!q || !kv8_pool || !kv8_scales || !out || (((uintptr_t)q | (uintptr_t)kv8_pool | (uintptr_t)kv8_scales | (uintptr_t)out) & 15) != 0 ||
        ((uintptr_t)lse & 3) != 0)
        return ASYNCLM_ERR_INVALID_ARG;
    if (!pages_chosen(plan)) return ASYNCLM_ERR_INVALID_ARG;
    if (int rc = check_plan_device(plan->device)) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    PlanUse use(plan, s);
    const cudaError_t e = use.dev.head_dim == 128 ? launch_kv8_d<128>(use.dev, q, kv8_pool, kv8_scales, out, lse, s)
                                                  : launch_kv8_d<64>(use.dev, q, kv8_pool, kv8_scales, out, lse, s);
    const int rc = cuda_status(use.launched(e));
    if (rc != ASYNCLM_OK) return rc;
    return cuda_status(launch_lse_merge(use.dev, out, lse, s));
}
