// The attention kernels' entry points and launchers.
//
// Three kernels are built from two bodies (attn_append_tc.cuh: span tiles on tcgen05, attn_decode.cuh: decode
// rows and short spans on warp-level MMAs):
//   attn_fused_kernel      a persistent CTA first runs its span items, then takes warp-body items
//                          (a CTA without span tiles skips the tensor-memory set-up altogether).
//                          One launch instead of two: the fixed cost of a launch (about 10 us of
//                          start-up and tail per kernel at 148 CTAs) is paid once, and a CTA that is
//                          done with its span tiles early moves on to decode rows at once.
//   attn_append_tc_kernel  steps that have span tiles only
//   attn_decode_kernel     steps without span tiles
// All are launched with programmatic stream serialization and wait for the kernel in front of them
// (normally the KV append) right before they first touch the pool.
#include "attn_append_tc.cuh"
#include "attn_decode.cuh"
#include "attn_launch.cuh"

namespace asynclm {

namespace {

template <int D, int G, bool APPEND>
__global__ void __launch_bounds__(dec::kThreads, 1)
attn_decode_kernel(DevPlan p, const __grid_constant__ CUtensorMap kv_map, const __nv_bfloat16* pool, const __nv_bfloat16* __restrict__ q,
                   __nv_bfloat16* __restrict__ out, float* __restrict__ lse, int S, AppendSrc app) {
    extern __shared__ uint8_t smem_raw[];
    pdl_trigger();      // the split-KV merge behind this kernel may start its prologue
    if (threadIdx.x == 0) { trace_mark(0); trace_set(1, 0); trace_set(5, 0); trace_set(6, 0); trace_set(7, 0); }
    dec::decode_body<D, G, APPEND, true>(p, &kv_map, pool, q, out, lse, S, aligned_smem(smem_raw), app);
}

template <int D, int G>
__global__ void __launch_bounds__(tc::kThreads, 1)
attn_append_tc_kernel(DevPlan p, const __grid_constant__ CUtensorMap span_map, const __nv_bfloat16* __restrict__ q, const __nv_bfloat16* pool,
                      __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
    extern __shared__ uint8_t smem_raw[];
    pdl_trigger();      // the kernel behind this one may start its prologue; it waits for this grid to complete
    if (threadIdx.x == 0) {
        trace_mark(0);
        for (int s = 8; s < 16; ++s) trace_set(s, 0);
    }
    tc::tc_body<D, G, true>(p, &span_map, q, pool, out, lse, aligned_smem(smem_raw));
    if (threadIdx.x == 0) trace_mark(1);
}

template <int D, int G>
__global__ void __launch_bounds__(tc::kThreads, 1)
attn_fused_kernel(DevPlan p, const __grid_constant__ CUtensorMap kv_map, const __grid_constant__ CUtensorMap span_map,
                  const __nv_bfloat16* __restrict__ q, const __nv_bfloat16* pool, __nv_bfloat16* __restrict__ out, float* __restrict__ lse,
                  int S) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = aligned_smem(smem_raw);
    pdl_trigger();      // the split-KV merge behind this kernel may start its prologue
    if (threadIdx.x == 0) { trace_mark(0); trace_set(1, 0); trace_set(5, 0); trace_set(6, 0); trace_set(7, 0); }
    const int32_t* head = p.cta_heads + (size_t)blockIdx.x * kHeadWords;
    // bring the whole header and the tensor map close now: the decode phase of a CTA that starts with
    // span tiles finds them in L2 when it gets there
    if (threadIdx.x < 3) asm volatile("prefetch.global.L2 [%0];" ::"l"(head + 32 * threadIdx.x));
    if (threadIdx.x == 32) asm volatile("prefetch.tensormap [%0];" ::"l"(&kv_map));
    if (head[0] == head[1]) {
        // no span tiles for this CTA: straight to its decode rows, without the tensor-memory set-up
        dec::decode_body<D, G, false, false>(p, &kv_map, nullptr, q, out, lse, S, smem, AppendSrc{});
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 8; s < 16; ++s) trace_set(s, 0);
    }
    tc::tc_body<D, G, false>(p, &span_map, q, pool, out, lse, smem);
    if (threadIdx.x == 0) trace_mark(1);
    if (head[2] == head[3] && p.queue_count == 0) return;      // nothing left for the warp body
    __syncthreads();      // tensor memory released, shared memory free for the second phase
    dec::decode_body<D, G, false, false>(p, &kv_map, nullptr, q, out, lse, S, smem, AppendSrc{});
}

template <int D, int G, bool APPEND>
cudaError_t launch_decode(const DevPlan& p, const void* q, const void* pool, void* out, float* lse,
                          cudaStream_t stream, AppendSrc app) {
    const int S = decode_stages<D>();
    const size_t smem = dec::smem_bytes<D>(S);
    cudaError_t e = allow_smem<attn_decode_kernel<D, G, APPEND>>(smem);
    if (e != cudaSuccess) return e;
    CUtensorMap map;
    if (p.num_pages > kMaxMapPages) return cudaErrorInvalidValue;
    e = pool_map(kKvMap, p, pool, &map);
    if (e != cudaSuccess) return e;
    return launch_when(!p.full_launch, attn_decode_kernel<D, G, APPEND>, dim3(p.num_ctas_cuda), dim3(dec::kThreads), smem, stream, p, map,
                      (const __nv_bfloat16*)pool, (const __nv_bfloat16*)q, (__nv_bfloat16*)out, lse, S, app);
}

template <int D, int G>
cudaError_t launch_tensor(const DevPlan& p, const void* q, const void* pool, void* out, float* lse, cudaStream_t stream) {
    constexpr size_t smem = tc::Geometry<D>::SMEM_BYTES;
    cudaError_t e = allow_smem<attn_append_tc_kernel<D, G>>(smem);
    if (e != cudaSuccess) return e;
    CUtensorMap map;
    e = pool_map(kSpanMap, p, pool, &map);
    if (e != cudaSuccess) return e;
    return launch_when(!p.full_launch, attn_append_tc_kernel<D, G>, dim3(p.num_ctas_tensor), dim3(tc::kThreads), smem, stream,
                      p, map, (const __nv_bfloat16*)q, (const __nv_bfloat16*)pool, (__nv_bfloat16*)out, lse);
}

template <int D, int G>
cudaError_t launch_fused(const DevPlan& p, const void* q, const void* pool, void* out, float* lse, cudaStream_t stream) {
    constexpr int S = decode_stages<D>();
    constexpr size_t smem = std::max<size_t>(dec::smem_bytes<D>(S), tc::Geometry<D>::SMEM_BYTES);
    static_assert(dec::smem_bytes<D>(S) - 1024 <= tc::Geometry<D>::OFF_BAR, "the span body's barriers stay clear of the warp body");
    cudaError_t e = allow_smem<attn_fused_kernel<D, G>>(smem);
    if (e != cudaSuccess) return e;
    CUtensorMap kv_map, span_map;
    if (p.num_pages > kMaxMapPages) return cudaErrorInvalidValue;
    e = pool_map(kKvMap, p, pool, &kv_map);
    if (e == cudaSuccess) e = pool_map(kSpanMap, p, pool, &span_map);
    if (e != cudaSuccess) return e;
    return launch_when(!p.full_launch, attn_fused_kernel<D, G>, dim3(p.num_ctas_cuda), dim3(tc::kThreads), smem, stream, p, kv_map, span_map,
                      (const __nv_bfloat16*)q, (const __nv_bfloat16*)pool, (__nv_bfloat16*)out, lse, S);
}

template <int D, int G>
cudaError_t launch_attention_impl(const DevPlan& p, const void* q, const void* kv_pool, void* out, float* lse,
                                  cudaStream_t stream, AppendSrc app) {
    const bool has_tensor = p.num_items_tensor > 0, has_cuda = p.num_items_cuda > 0;
    if (app.k_new != nullptr)      // the warp body only
        return has_tensor || !has_cuda ? cudaErrorInvalidValue : launch_decode<D, G, true>(p, q, kv_pool, out, lse, stream, app);
    if (has_tensor && has_cuda && p.num_ctas_tensor == p.num_ctas_cuda)
        return launch_fused<D, G>(p, q, kv_pool, out, lse, stream);
    if (has_tensor)
        if (cudaError_t e = launch_tensor<D, G>(p, q, kv_pool, out, lse, stream)) return e;
    // a decode kernel behind a tensor kernel would have to wait for it to finish (pdl_wait), which is what
    // stream order gives anyway
    return has_cuda ? launch_decode<D, G, false>(p, q, kv_pool, out, lse, stream, app) : cudaSuccess;
}

template <int D>
cudaError_t launch_attention_d(const DevPlan& p, const void* q, const void* kv_pool, void* out, float* lse,
                               cudaStream_t stream, AppendSrc app) {
    switch (p.group) {
        case 1: return launch_attention_impl<D, 1>(p, q, kv_pool, out, lse, stream, app);
        case 2: return launch_attention_impl<D, 2>(p, q, kv_pool, out, lse, stream, app);
        case 4: return launch_attention_impl<D, 4>(p, q, kv_pool, out, lse, stream, app);
        case 8: return launch_attention_impl<D, 8>(p, q, kv_pool, out, lse, stream, app);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace

cudaError_t launch_attention(const DevPlan& p, const void* q, const void* kv_pool, void* out, float* lse,
                             cudaStream_t stream, AppendSrc app) {
    if (p.head_dim == 128) return launch_attention_d<128>(p, q, kv_pool, out, lse, stream, app);
    if (p.head_dim == 64) return launch_attention_d<64>(p, q, kv_pool, out, lse, stream, app);
    return cudaErrorInvalidValue;
}

}  // namespace asynclm

#ifdef ASYNCLM_TRACE
// Debug builds only: copies the per-CTA time stamps of the last attention launch to the host
// (synchronises the device).  out: [1024][8] unsigned 64-bit.
extern "C" int asynclm_trace_read(unsigned long long* out) {
    return cudaMemcpyFromSymbol(out, asynclm::g_trace, sizeof(asynclm::g_trace)) == cudaSuccess ? 0 : -5;
}
// The event log of the first CTAs: out [4][11][512] unsigned 64-bit (cycle << 8 | event); clears it.
extern "C" int asynclm_trace_events_read(unsigned long long* out) {
    if (cudaMemcpyFromSymbol(out, asynclm::g_events, sizeof(asynclm::g_events)) != cudaSuccess) return -5;
    void* dev = nullptr;
    if (cudaGetSymbolAddress(&dev, asynclm::g_events) != cudaSuccess) return -5;
    return cudaMemset(dev, 0, sizeof(asynclm::g_events)) == cudaSuccess ? 0 : -5;
}
#endif