// Which pages a token attends to: for every (token, kv head) the first and the last pages that it sees and, up to the budget, those whose keys
// could score highest.
//
// Score.  For a query q and a page whose keys lie between lo and hi, channel by channel, no key scores more than
//     sum_c max(q_c lo_c, q_c hi_c) = sum_c q_c (q_c < 0 ? lo_c : hi_c);
// a page's score is the largest over the G queries of the kv head.  Two sums of 32 bits in different orders differ in their last bits, and with
// them the choice, wherever two pages are close.  So the sums are held in 64 bits, where a product of bf16 values is exact: the choice depends on
// the values alone but for ties within 2^-45.  A bf16 value becomes an fp64 one by its bits (the upper word holds all of it), and which of lo and hi
// is wanted is a bit operation on that word.
//
// A CTA scores kSelectChunkPages pages of one (row, kv head), a warp 16 / G of them at a time, four channels to a lane; the 16 sums are exchanged
// and halved together.  Scores go to the workspace as ordered integers.  The CTA that finishes a row's last chunk selects: the 64-bit threshold
// by histograms of eight bits, from the first bit in which the scores differ, then the pages in rising order, each thread a stretch of them.
#include <algorithm>

#include "asynclm.h"
#include "common.cuh"
#include "kernels.h"
#include "plan_internal.h"

namespace asynclm {

namespace {

constexpr int kSelectThreads = 256, kSelectWarps = kSelectThreads / 32;
constexpr int kKeysInShared = 4096;      // of a row (65 536 tokens); longer ones are read from L2
constexpr unsigned long long kAlways = ~0ull;      // key of a page that is taken whatever its score

// Upper word of the fp64 number with a bf16 number's value (the lower word is zero).  Subnormal ones count as zero, infinities and NaN as 2^128 and
// more, with their sign.
__device__ __forceinline__ uint32_t f64_word(uint32_t bf16_bits) {
    const uint32_t m = bf16_bits & 0x7fffu;
    return m < 0x80u ? 0u : (bf16_bits & 0x8000u) << 16 | ((m << 13) + 0x38000000u);
}
__device__ __forceinline__ double f64_of(uint32_t word) { return __hiloint2double((int)word, 0); }

__device__ __forceinline__ unsigned long long ordered(double x) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}

template <int D, int G>
struct SelectShape {
    static constexpr int LANES = D / 4;              // of a page: four channels to a lane
    static constexpr int AT_ONCE = 32 / LANES;       // pages that a warp's load covers
    static constexpr int LOADS = 16 / G;             // of them, together 16 sums a lane
    static constexpr int PAGES = LOADS * AT_ONCE;
};

// Sums v[0 .. 15] over the lanes of a page (LANES of them, next to each other); lane l gets sum number index16(l).
template <int LANES>
__device__ __forceinline__ double reduce16(double (&v)[16], int lane) {
#pragma unroll
    for (int half = 8; half >= 1; half >>= 1) {
        const int bit = LANES / 16 * half;
        const bool upper = (lane & bit) != 0;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const double send = upper ? v[i] : v[i + half], keep = upper ? v[i + half] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
        }
    }
    return LANES == 32 ? v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1) : v[0];
}

template <int D, int G>
__global__ void __launch_bounds__(kSelectThreads)
select_pages_kernel(DevPlan p, const uint8_t* __restrict__ q, const uint8_t* __restrict__ bounds, int32_t* __restrict__ pages_out) {
    using S = SelectShape<D, G>;
    __shared__ unsigned long long s_keys[kKeysInShared];
    __shared__ int s_hist[256];
    __shared__ unsigned long long s_lo[kSelectWarps], s_hi[kSelectWarps];
    __shared__ int s_count[kSelectWarps][2];
    __shared__ int s_bin, s_above, s_in, s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int h = blockIdx.x % p.num_kv_heads;
    const SelectChunk c = p.select_chunks[blockIdx.x / p.num_kv_heads];
    const int row = c.row, seq = __ldg(p.row_seq + row);
    const int np = (__ldg(p.kv_len_before + seq) + row - __ldg(p.q_indptr + seq)) / kPage + 1;      // pages that the token sees
    const int32_t* table = p.page_indices + __ldg(p.page_indptr + seq);
    const int budget = p.select_budget;
    const size_t pair = (size_t)row * p.num_kv_heads + h;
    int32_t* list = p.select_pages + pair * budget;
    int32_t* out = pages_out == nullptr ? nullptr : pages_out + pair * budget;
    pdl_wait();      // queries and bounds are the kernels' in front, and so are the lists as long as the last attention reads them
    if (np <= budget) {
        for (int j = tid; j < budget; j += kSelectThreads) {
            if (j < np) list[j] = __ldg(table + j);
            if (out != nullptr) out[j] = j < np ? j : -1;
        }
        return;
    }
    unsigned long long* keys = p.select_keys + p.select_base[row] * p.num_kv_heads + (size_t)h * np;
    // ---- scores
    {
        uint32_t qw[G][4], neg[G][4];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uint2 w = *reinterpret_cast<const uint2*>(q + (((size_t)row * p.num_q_heads + (size_t)h * G + g) * D + (size_t)(lane % S::LANES) * 4) * 2);
            const uint32_t x[4] = {w.x & 0xffffu, w.x >> 16, w.y & 0xffffu, w.y >> 16};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                qw[g][i] = f64_word(x[i]);
                neg[g][i] = (uint32_t)((int32_t)qw[g][i] >> 31);
            }
        }
        const int end = min(c.page0 + kSelectChunkPages, np);
        for (int j0 = c.page0 + warp * S::PAGES; j0 < end; j0 += kSelectWarps * S::PAGES) {
            uint2 wl[S::LOADS], wh[S::LOADS];
#pragma unroll
            for (int u = 0; u < S::LOADS; ++u) {
                const int j = min(j0 + u * S::AT_ONCE + lane / S::LANES, end - 1);
                const uint8_t* src = bounds + (((size_t)__ldg(table + j) * p.num_kv_heads + h) * 2) * D * 2 + (size_t)(lane % S::LANES) * 8;
                wl[u] = *reinterpret_cast<const uint2*>(src);
                wh[u] = *reinterpret_cast<const uint2*>(src + D * 2);
            }
            double v[16];
#pragma unroll
            for (int u = 0; u < S::LOADS; ++u) {
#pragma unroll
                for (int g = 0; g < G; ++g) v[u * G + g] = 0.0;
                const uint32_t l[4] = {wl[u].x & 0xffffu, wl[u].x >> 16, wl[u].y & 0xffffu, wl[u].y >> 16};
                const uint32_t t[4] = {wh[u].x & 0xffffu, wh[u].x >> 16, wh[u].y & 0xffffu, wh[u].y >> 16};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t lo = f64_word(l[i]), hi = f64_word(t[i]), differ = lo ^ hi;
#pragma unroll
                    for (int g = 0; g < G; ++g) v[u * G + g] = fma(f64_of(qw[g][i]), f64_of(hi ^ (differ & neg[g][i])), v[u * G + g]);
                }
            }
            double s = reduce16<S::LANES>(v, lane);
            // the largest over the heads: their number is the low bits of the sum's
            constexpr int kUnit = S::LANES / 16;
#pragma unroll
            for (int off = kUnit; off < kUnit * G; off <<= 1) s = fmax(s, __shfl_xor_sync(0xffffffffu, s, off));
            const int number = lane % S::LANES / kUnit, j = j0 + number / G * S::AT_ONCE + lane / S::LANES;
            if (lane % kUnit == 0 && number % G == 0 && j < end) {
                const bool always = j < p.select_first || j >= np - p.select_last;
                keys[j] = always ? kAlways : ordered(s);
            }
        }
    }
    // ---- the CTA that completes the row goes on
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        const int chunks = (np + kSelectChunkPages - 1) / kSelectChunkPages;
        s_last = atomicAdd(p.select_arrivals + pair, 1) == chunks - 1;
        if (s_last) {
            p.select_arrivals[pair] = 0;      // ready for the next launch
            __threadfence();
        }
    }
    __syncthreads();
    if (!s_last) return;
    const bool shared = np <= kKeysInShared;
    unsigned long long lo = ~0ull, hi = 0;      // of the scores
    for (int j = tid; j < np; j += kSelectThreads) {
        const unsigned long long k = __ldcg(keys + j);
        if (shared) s_keys[j] = k;
        if (k != kAlways) lo = min(lo, k), hi = max(hi, k);
    }
    auto key = [&](int j) { return shared ? s_keys[j] : __ldcg(keys + j); };
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, off));
        hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, off));
    }
    if (lane == 0) s_lo[warp] = lo, s_hi[warp] = hi;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelectWarps; ++w) lo = min(lo, s_lo[w]), hi = max(hi, s_hi[w]);
    // ---- threshold: keys above `hi` are in, below `lo` out, and of those in between the first `need` pages
    int need = budget - p.select_first - p.select_last;
    if (need == 0) {
        lo = kAlways, hi = kAlways - 1;
    } else {
        int shift = lo == hi ? 0 : max(0, 56 - __clzll((long long)(lo ^ hi)));
        while (true) {
            const unsigned long long base = lo >> shift;
            s_hist[tid] = 0;
            __syncthreads();
            for (int j = tid; j < np; j += kSelectThreads) {
                const unsigned long long k = key(j);
                if (k >= lo && k <= hi) atomicAdd(&s_hist[(int)((k >> shift) - base)], 1);
            }
            __syncthreads();
            if (warp == 0) {      // a lane takes eight bins, the highest lane the highest
                int n[8], sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) n[i] = s_hist[8 * lane + i], sum += n[i];
                int above = sum;      // in this lane's bins and all higher ones
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const int more = __shfl_down_sync(0xffffffffu, above, off);
                    if (lane + off < 32) above += more;
                }
                above -= sum;
                if (above < need && need <= above + sum) {
                    int i = 7;
                    while (above + n[i] < need) above += n[i], --i;
                    s_bin = 8 * lane + i;
                    s_above = above;
                    s_in = n[i];
                }
            }
            __syncthreads();
            need -= s_above;
            const unsigned long long first = (base + (unsigned)s_bin) << shift, last = first + ((1ull << shift) - 1);
            lo = max(lo, first);
            hi = min(hi, last);
            if (s_in == need || shift == 0) break;
            shift = max(0, shift - 8);
            __syncthreads();      // (s_bin is read before it is written again)
        }
    }
    // ---- the list: a stretch of pages to a thread
    const int per = (np + kSelectThreads - 1) / kSelectThreads, first = min(tid * per, np), last = min(first + per, np);
    int above = 0, among = 0;
    for (int j = first; j < last; ++j) {
        const unsigned long long k = key(j);
        above += k > hi;
        among += k >= lo && k <= hi;
    }
    int before_above = above, before_among = among;      // inclusive sums, then those of the threads in front
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int a = __shfl_up_sync(0xffffffffu, before_above, off), b = __shfl_up_sync(0xffffffffu, before_among, off);
        if (lane >= off) before_above += a, before_among += b;
    }
    if (lane == 31) s_count[warp][0] = before_above, s_count[warp][1] = before_among;
    __syncthreads();
    before_above -= above;
    before_among -= among;
    for (int w = 0; w < warp; ++w) before_above += s_count[w][0], before_among += s_count[w][1];
    for (int j = first; j < last; ++j) {
        const unsigned long long k = key(j);
        const bool in = k >= lo && k <= hi;
        if (k > hi || (in && before_among < need)) {
            const int at = before_above + min(before_among, need);
            list[at] = __ldg(table + j);
            if (out != nullptr) out[at] = j;
        }
        before_above += k > hi;
        before_among += in;
    }
}

template <int D>
cudaError_t launch_select(const DevPlan& p, const void* q, const void* bounds, int32_t* pages_out, cudaStream_t s) {
    const dim3 grid((unsigned)(p.num_select_chunks * p.num_kv_heads));
    auto kernel = p.group == 1 ? select_pages_kernel<D, 1> : p.group == 2 ? select_pages_kernel<D, 2> : p.group == 4 ? select_pages_kernel<D, 4>
                                                                                                                     : select_pages_kernel<D, 8>;
    return launch_when(!p.full_launch, kernel, grid, dim3(kSelectThreads), 0, s, p, (const uint8_t*)q, (const uint8_t*)bounds, pages_out);
}

}  // namespace

}  // namespace asynclm

extern "C" int asynclm_select_pages(const asynclm_plan_t* plan, const void* q, const void* key_bounds, int32_t* pages_out, void* stream) {
    using namespace asynclm;
    if (!plan || plan->magic != kPlanMagic || plan->host_only || !plan->sparse) return ASYNCLM_ERR_INVALID_ARG;
    if (plan->dev.total_q == 0) return ASYNCLM_OK;
    if (!q || !key_bounds || (((uintptr_t)q | (uintptr_t)key_bounds) & 15) != 0 || ((uintptr_t)pages_out & 3) != 0) return ASYNCLM_ERR_INVALID_ARG;
    if (int rc = check_plan_device(plan->device)) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    PlanUse use(plan, s);
    const cudaError_t e = use.dev.head_dim == 128 ? launch_select<128>(use.dev, q, key_bounds, pages_out, s) : launch_select<64>(use.dev, q, key_bounds, pages_out, s);
    const int rc = cuda_status(use.launched(e));
    if (rc == ASYNCLM_OK) __atomic_store_n(&plan->selected, 1, __ATOMIC_RELEASE);
    return rc;
}
