// Rotary positions of query and key rows, for caches that stay in bf16 (the fused form for the 8-bit cache is
// kv8_append.cu; the mathematics and the division among threads are in rope_rows.cuh), and the table of frequencies
// that both take.
#include <math.h>

#include <algorithm>
#include <cstring>

#include "kernels.h"
#include "rope_rows.cuh"

namespace asynclm {

namespace {

constexpr int32_t kRopeMagic = 0x45504f52;      // "ROPE"
constexpr double kTwoPi = 6.283185307179586476925286766559;

struct RopeSets { RowSet set[2]; };

// Grid: one CTA for `tokens` tokens; its warps take blocks of rows of one token, and request the next block's rows
// before they turn one's.
template <int FORM>
__global__ void __launch_bounds__(kRopeRowThreads, rope_ctas(FORM))
rope_apply_kernel(const __grid_constant__ RopeTurns turns, const __grid_constant__ RopeSets sets, const int32_t* positions, int total, int head_dim, int tokens) {
    extern __shared__ uint4 smem[];
    float4 (*table)[kRopeEntries] = reinterpret_cast<float4 (*)[kRopeEntries]>(smem + kRopeRowThreads);
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int per_row = head_dim / 8, rows = 32 / per_row;      // lanes of a row, rows of a warp
    const int v = lane % per_row, sub = lane / per_row;
    const int r0 = blockIdx.x * tokens, n = min(tokens, total - r0);
    const int block = rows * kRopeUnroll;
    const int blocks0 = (sets.set[0].heads + block - 1) / block, blocks = blocks0 + (sets.set[1].heads + block - 1) / block;
    struct Block { uint4 x[kRopeUnroll]; };
    auto load = [&](int item) {
        Block l;
        const int i = item / blocks, b = item % blocks;
        const RowSet& set = sets.set[b < blocks0 ? 0 : 1];
        const int h0 = (b < blocks0 ? b : b - blocks0) * block + sub;
        const __nv_bfloat16* in = set.in + (int64_t)(r0 + i) * set.in_stride + 8 * v;
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u)
            l.x[u] = item < n * blocks && sub < rows && h0 + u * rows < set.heads ? __ldcg(reinterpret_cast<const uint4*>(in + (int64_t)(h0 + u * rows) * head_dim))
                                                                                 : make_uint4(0, 0, 0, 0);
        return l;
    };
    pdl_wait();      // rows and positions belong to the kernels in front until those have completed
    Block next = load(warp);
    rope_fill<FORM>(turns, table, n, [&](int i) { return __ldcg(positions + r0 + i); });
    __syncthreads();
    for (int item = warp; item < n * blocks; item += warps) {
        const Block now = next;
        next = load(item + warps);
        const int i = item / blocks, b = item % blocks;
        const RowSet& set = sets.set[b < blocks0 ? 0 : 1];
        const int h0 = (b < blocks0 ? b : b - blocks0) * block + sub;
        __nv_bfloat16* out = set.out + (int64_t)(r0 + i) * set.out_stride + 8 * v;
        const RopeLane<FORM> cs = rope_lane<FORM>(turns, table[i], v);
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
            float y[8];
            rope_turn<FORM>(turns, cs, v, lane, smem + warp * 32, now.x[u], y);
            const uint4 o = rope_words<FORM>(turns, v, now.x[u], y);
            if (sub < rows && h0 + u * rows < set.heads) *reinterpret_cast<uint4*>(out + (int64_t)(h0 + u * rows) * head_dim) = o;
        }
    }
}

}  // namespace

bool rope_turns(const asynclm_rope_table* table, int head_dim, RopeTurns* out) {
    if (table->magic != kRopeMagic || table->head_dim != head_dim || table->rotary_dim < 2 || table->rotary_dim > head_dim || table->rotary_dim % 2 != 0)
        return false;
    std::memcpy(out->turns, table->turns, sizeof(out->turns));
    out->factor = table->factor;
    out->rotary_dim = table->rotary_dim;
    out->layout = table->layout;
    return true;
}

}  // namespace asynclm

using namespace asynclm;

extern "C" int asynclm_rope_table_init(const asynclm_rope* rope, int32_t head_dim, asynclm_rope_table* out) {
    if (!rope || !out || head_dim < 8 || head_dim > 2 * kRopeMaxPairs || head_dim % 8 != 0) return ASYNCLM_ERR_INVALID_ARG;
    const int rd = rope->rotary_dim == 0 ? head_dim : rope->rotary_dim;
    if (rd < 2 || rd > head_dim || rd % 2 != 0 || !(rope->theta > 1.0) || !std::isfinite(rope->theta)) return ASYNCLM_ERR_INVALID_ARG;
    if (rope->layout != ASYNCLM_ROPE_HALF && rope->layout != ASYNCLM_ROPE_INTERLEAVED) return ASYNCLM_ERR_INVALID_ARG;
    const int scaling = rope->scaling;
    if (scaling < ASYNCLM_ROPE_UNSCALED || scaling > ASYNCLM_ROPE_YARN) return ASYNCLM_ERR_INVALID_ARG;
    const double s = scaling == ASYNCLM_ROPE_UNSCALED ? 1.0 : rope->factor, context = (double)rope->context;
    if (!(s >= 1.0) || !std::isfinite(s)) return ASYNCLM_ERR_INVALID_ARG;
    if (scaling >= ASYNCLM_ROPE_BANDS && rope->context <= 0) return ASYNCLM_ERR_INVALID_ARG;
    const double low = rope->low_freq_factor, high = rope->high_freq_factor;
    if (scaling == ASYNCLM_ROPE_BANDS && !(low > 0.0 && high > low && std::isfinite(high))) return ASYNCLM_ERR_INVALID_ARG;
    double first = 0.0, last = 0.0, factor = 1.0;
    if (scaling == ASYNCLM_ROPE_YARN) {
        if (!(rope->beta_slow > 0.0 && rope->beta_fast > rope->beta_slow && std::isfinite(rope->beta_fast)) || !(rope->attention_factor >= 0.0))
            return ASYNCLM_ERR_INVALID_ARG;
        // the pair that turns `beta` times over the context: theta^(-2j / rd) * context = 2 pi beta
        auto pair = [&](double beta) { return rd * std::log(context / (kTwoPi * beta)) / (2.0 * std::log(rope->theta)); };
        first = std::max(std::floor(pair(rope->beta_fast)), 0.0);
        last = std::min(std::ceil(pair(rope->beta_slow)), (double)(rd - 1));
        factor = rope->attention_factor > 0.0 ? rope->attention_factor : 0.1 * std::log(s) + 1.0;
    }
    std::memset(out, 0, sizeof(*out));
    for (int j = 0; j < rd / 2; ++j) {
        double f = std::pow(rope->theta, -2.0 * j / rd);
        if (scaling == ASYNCLM_ROPE_LINEAR) f /= s;
        if (scaling == ASYNCLM_ROPE_BANDS) {
            // turns over the context: above `high` the pair is left alone, below `low` its positions are divided by s
            const double kept = std::min(std::max((context * f / kTwoPi - low) / (high - low), 0.0), 1.0);
            f = (1.0 - kept) * f / s + kept * f;
        }
        if (scaling == ASYNCLM_ROPE_YARN) {
            const double divided = std::min(std::max((j - first) / std::max(last - first, 1e-3), 0.0), 1.0);
            f = divided * f / s + (1.0 - divided) * f;
        }
        out->turns[j] = f / kTwoPi;
    }
    out->magic = kRopeMagic;
    out->head_dim = head_dim;
    out->rotary_dim = rd;
    out->layout = rope->layout;
    out->factor = factor;
    return ASYNCLM_OK;
}

extern "C" int asynclm_rope_apply(const asynclm_rope_table* table, const int32_t* positions, int32_t tokens, int32_t head_dim,
                                  const asynclm_rope_rows* rows, int32_t n_rows, void* stream) {
    if (!table || !rows || n_rows < 1 || n_rows > 2 || tokens < 0) return ASYNCLM_ERR_INVALID_ARG;
    RopeTurns turns;
    if (!rope_turns(table, head_dim, &turns)) return ASYNCLM_ERR_INVALID_ARG;
    RopeSets sets{};
    for (int k = 0; k < n_rows; ++k) {
        const asynclm_rope_rows& r = rows[k];
        const int64_t dense = (int64_t)r.heads * head_dim;
        const int64_t si = r.in_stride == 0 ? dense : r.in_stride, so = r.out_stride == 0 ? dense : r.out_stride;
        if (r.heads < 1 || r.heads > (1 << 16) || si < dense || so < dense || si % 8 != 0 || so % 8 != 0) return ASYNCLM_ERR_INVALID_ARG;
        if (tokens > 0 && (!r.in || !r.out || (((uintptr_t)r.in | (uintptr_t)r.out) & 15) != 0 || (r.in == r.out && si != so))) return ASYNCLM_ERR_INVALID_ARG;
        sets.set[k] = RowSet{(const __nv_bfloat16*)r.in, (__nv_bfloat16*)r.out, si, so, r.heads, 1};
    }
    if (tokens == 0) return ASYNCLM_OK;
    if (!positions || ((uintptr_t)positions & 3) != 0) return ASYNCLM_ERR_INVALID_ARG;
    const int per_cta = rope_row_tokens(tokens, rope_form(turns));
    const int block = 32 / (head_dim / 8) * kRopeUnroll;
    const int blocks = (sets.set[0].heads + block - 1) / block + (sets.set[1].heads + block - 1) / block;
    const int threads = 32 * std::min(kRopeRowThreads / 32, per_cta * blocks);
    const auto launch = [&](auto kernel) {
        return cuda_status(launch_pdl(kernel, dim3((tokens + per_cta - 1) / per_cta), dim3(threads), rope_row_smem(per_cta), (cudaStream_t)stream, turns, sets,
                                      positions, tokens, head_dim, per_cta));
    };
    switch (rope_form(turns)) {
        case kRopeHalves: return launch(rope_apply_kernel<kRopeHalves>);
        case kRopePairs: return launch(rope_apply_kernel<kRopePairs>);
        case kRopeOddPairs: return launch(rope_apply_kernel<kRopeOddPairs>);
        default: return launch(rope_apply_kernel<kRopeOddHalves>);
    }
}
