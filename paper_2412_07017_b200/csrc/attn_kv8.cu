// Attention over the 8-bit cache: the entry point, its kernels and launcher.  The bodies are those of the bf16 cache, with the cache's
// format as a template parameter (attn_decode.cuh: what a consumer warp does with a page).
#include "asynclm.h"
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

template <int D, int G>
cudaError_t launch_kv8_impl(const DevPlan& p, const void* q, const void* pool, const void* scales, void* out, float* lse, cudaStream_t stream) {
    if (p.num_items_tensor > 0) return cudaErrorNotSupported;
    if (p.num_items_cuda == 0) return cudaSuccess;
    if (p.num_pages > kMaxMapPages) return cudaErrorInvalidValue;
    constexpr int S = decode_stages<D, true>();
    constexpr size_t smem = dec::smem_bytes<D, true>(S);
    cudaError_t e = allow_smem<attn_decode_kv8_kernel<D, G>>(smem);
    if (e != cudaSuccess) return e;
    CUtensorMap map;
    e = pool_map(kKv8Map, p, pool, &map);
    if (e != cudaSuccess) return e;
    return launch_when(!p.full_launch, attn_decode_kv8_kernel<D, G>, dim3(p.num_ctas_cuda), dim3(dec::kThreads), smem, stream, p, map, (const uint8_t*)pool,
                       (const uint8_t*)scales, (const __nv_bfloat16*)q, (__nv_bfloat16*)out, lse, S);
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
    if (int rc = check_plan_device(plan->device)) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    PlanUse use(plan, s);
    const cudaError_t e = use.dev.head_dim == 128 ? launch_kv8_d<128>(use.dev, q, kv8_pool, kv8_scales, out, lse, s)
                                                  : launch_kv8_d<64>(use.dev, q, kv8_pool, kv8_scales, out, lse, s);
    const int rc = cuda_status(use.launched(e));
    if (rc != ASYNCLM_OK) return rc;
    return cuda_status(launch_lse_merge(use.dev, out, lse, s));
}
