// The append of the 8-bit cache: the step's new K and V rows, quantised as they are written into their page slots, the
// keys (and, if asked, the queries) turned by their positions on the way.
//
// The interrupt block goes to the end of the context (paper Section 3.2): new token i of sequence b sits at position
// ctx_b + i, in the slot that the planner resolved.  A row is read once, turned in fp32 (rope_rows.cuh), its largest
// magnitude found by shuffles over the head_dim / 8 lanes that hold it, and its codes and scale written (kv8.cuh):
// there is one rounding between the projection's bf16 and the code. It moves 3 d bytes for a K or V row and 4 d for a
// query row, in whole 128-byte lines at head_dim 128.  8192 tokens of 32 / 8 heads of 128, queries too, 64 values of a
// row rotated, take 46.7 us, 4.0 TB/s: bound by instructions (72 % of the issue slots; the rotation in two parts,
// maxima and conversions); few tokens by launch and latency, 3.6 us in a graph.
#include <algorithm>

#include "kernels.h"
#include "plan_internal.h"
#include "rope_rows.cuh"

namespace asynclm {

namespace {

struct AppendSets { RowSet set[3]; };      // K, V, Q

template <int FORM>
__global__ void __launch_bounds__(kRopeRowThreads, rope_ctas(FORM))
kv8_append_kernel(DevPlan p, const __grid_constant__ RopeTurns turns, const __grid_constant__ AppendSets sets, uint8_t* pool, uint8_t* scales, int tokens) {
    extern __shared__ uint4 smem[];
    float4 (*table)[kRopeEntries] = reinterpret_cast<float4 (*)[kRopeEntries]>(smem + kRopeRowThreads);
    pdl_trigger();   // the attention kernel may start its prologue; it waits for this grid before reading the pool
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int d = p.head_dim, hkv = p.num_kv_heads;
    const int per_row = d / 8, rows = 32 / per_row;      // lanes of a row (16 or 8), rows of a warp
    const int v = lane % per_row, sub = lane / per_row;
    const int r0 = blockIdx.x * tokens, n = min(tokens, p.total_q - r0);
    const int block = rows * kRopeUnroll;
    const int blocks_kv = (hkv + block - 1) / block, blocks = 2 * blocks_kv + (sets.set[2].heads + block - 1) / block;
    auto kind = [&](int b) { return b < blocks_kv ? 0 : b < 2 * blocks_kv ? 1 : 2; };      // K, V, Q
    struct Block { uint4 x[kRopeUnroll]; };
    auto load = [&](int item) {
        Block l;
        const int i = item / blocks, b = item % blocks, which = kind(b);
        const RowSet& set = sets.set[which];
        const int h0 = (b - which * blocks_kv) * block + sub;
        const __nv_bfloat16* in = set.in + (int64_t)(r0 + i) * set.in_stride + 8 * v;
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u)
            l.x[u] = item < n * blocks && h0 + u * rows < set.heads ? __ldcg(reinterpret_cast<const uint4*>(in + (int64_t)(h0 + u * rows) * d)) : make_uint4(0, 0, 0, 0);
        return l;      // (not through the read-only path: q_out may be q itself)
    };
    // The angles come from the plan, which is there when this kernel starts (see PlanUse); rows and pool belong to the
    // kernels in front until those have completed.  Where all CTAs start at once the angles overlap the tail of the
    // kernel in front; in a longer grid the first rows are requested in front of them.
    const bool rows_first = gridDim.x > 148 * 2;
    Block next;
    if (rows_first) {
        pdl_wait();
        next = load(warp);
    }
    rope_fill<FORM>(turns, table, n, [&](int i) {
        const int r = r0 + i, b = __ldg(p.row_seq + r);
        return __ldg(p.kv_len_before + b) + r - __ldg(p.q_indptr + b);
    });
    if (!rows_first) {
        pdl_wait();
        next = load(warp);
    }
    __syncthreads();
    for (int item = warp; item < n * blocks; item += warps) {
        const Block now = next;
        next = load(item + warps);
        const int i = item / blocks, b = item % blocks, which = kind(b);
        const RowSet& set = sets.set[which];
        const int h0 = (b - which * blocks_kv) * block + sub;
        const int64_t slot = which < 2 ? __ldg(p.row_slot + r0 + i) : 0;
        RopeLane<FORM> cs;
        const bool turned = set.turned != 0 && turns.rotary_dim > 0;
        if (turned) cs = rope_lane<FORM>(turns, table[i], v);
        const bool page_fine = which == 2 || page_ok(slot / kPage, p.num_pages, p.status, kStatusBadPageAppend);
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
            const int h = h0 + u * rows;
            const bool on = h < set.heads;
            const uint4 x = now.x[u];
            float y[8];
            if (turned) {
                rope_turn<FORM>(turns, cs, v, lane, smem + warp * 32, x, y);
            } else {
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) { y[2 * k] = bf16_lo(w[k]); y[2 * k + 1] = bf16_hi(w[k]); }
            }
            if (which == 2) {
                if (on) {
                    const uint4 o = rope_words<FORM>(turns, v, x, y);
                    *reinterpret_cast<uint4*>(set.out + (int64_t)(r0 + i) * set.out_stride + (int64_t)h * d + 8 * v) = o;
                }
                continue;
            }
            uint32_t most = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) most = max(most, __float_as_uint(y[k]) & 0x7fffffffu);
            for (int off = 1; off < per_row; off <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
            const uint32_t byte = kv8_scale_byte(most);
            const float inv = byte == kKv8NanByte ? 0.f : __uint_as_float((254u - byte) << 23);      // 2^-e
            uint2 codes = make_uint2(kv8_encode2(y[0] * inv, y[1] * inv) | kv8_encode2(y[2] * inv, y[3] * inv) << 16,
                                     kv8_encode2(y[4] * inv, y[5] * inv) | kv8_encode2(y[6] * inv, y[7] * inv) << 16);
            if (byte == kKv8NanByte) codes = make_uint2(0, 0);
            if (on && page_fine) {
                *reinterpret_cast<uint2*>(pool + kv8_row_offset(slot / kPage, which, h, (int)(slot % kPage), hkv, d) + 8 * v) = codes;
                if (v == 0) scales[kv8_scale_offset(slot / kPage, which, h, (int)(slot % kPage), hkv)] = (uint8_t)byte;
            }
        }
    }
}

}  // namespace

}  // namespace asynclm

extern "C" int asynclm_kv8_append(const asynclm_plan_t* plan, const asynclm_kv8_rows* rows, void* kv8_pool, void* kv8_scales,
                                  const asynclm_rope_table* rope, void* stream) {
    using namespace asynclm;
    if (!plan || plan->magic != kPlanMagic || plan->host_only || !rows) return ASYNCLM_ERR_INVALID_ARG;
    const DevPlan& d = plan->dev;
    RopeTurns turns{};
    if (rope && !rope_turns(rope, d.head_dim, &turns)) return ASYNCLM_ERR_INVALID_ARG;
    if ((rows->q != nullptr) != (rows->q_out != nullptr) || (rows->q && !rope)) return ASYNCLM_ERR_INVALID_ARG;
    const int64_t kv = (int64_t)d.num_kv_heads * d.head_dim, qd = (int64_t)d.num_q_heads * d.head_dim;
    const int64_t ks = rows->k_stride ? rows->k_stride : kv, vs = rows->v_stride ? rows->v_stride : kv, qs = rows->q_stride ? rows->q_stride : qd;
    if (ks < kv || vs < kv || qs < qd || ((ks | vs | qs) & 7) != 0) return ASYNCLM_ERR_INVALID_ARG;
    if (rows->q && rows->q == rows->q_out && qs != qd) return ASYNCLM_ERR_INVALID_ARG;      // (q_out is dense)
    if (d.total_q == 0) return ASYNCLM_OK;
    if (!rows->k || !rows->v || !kv8_pool || !kv8_scales ||
        (((uintptr_t)rows->k | (uintptr_t)rows->v | (uintptr_t)rows->q | (uintptr_t)rows->q_out | (uintptr_t)kv8_pool | (uintptr_t)kv8_scales) & 15) != 0)
        return ASYNCLM_ERR_INVALID_ARG;
    if (int rc = check_plan_device(plan->device)) return rc;
    AppendSets sets{};
    sets.set[0] = RowSet{(const __nv_bfloat16*)rows->k, nullptr, ks, 0, d.num_kv_heads, 1};
    sets.set[1] = RowSet{(const __nv_bfloat16*)rows->v, nullptr, vs, 0, d.num_kv_heads, 0};
    if (rows->q) sets.set[2] = RowSet{(const __nv_bfloat16*)rows->q, (__nv_bfloat16*)rows->q_out, qs, qd, d.num_q_heads, 1};
    PlanUse use(plan, (cudaStream_t)stream);
    const int tokens = rope_row_tokens(d.total_q, rope_form(turns)), block = 32 / (d.head_dim / 8) * kRopeUnroll;
    const int blocks = 2 * ((d.num_kv_heads + block - 1) / block) + (sets.set[2].heads + block - 1) / block;
    const int threads = 32 * std::min(kRopeRowThreads / 32, tokens * blocks);
    const auto launch = [&](auto kernel) {
        return cuda_status(use.launched(launch_when(!use.dev.full_launch, kernel, dim3((d.total_q + tokens - 1) / tokens), dim3(threads), rope_row_smem(tokens),
                                                    (cudaStream_t)stream, use.dev, turns, sets, (uint8_t*)kv8_pool, (uint8_t*)kv8_scales, tokens)));
    };
    switch (rope_form(turns)) {
        case kRopeHalves: return launch(kv8_append_kernel<kRopeHalves>);
        case kRopePairs: return launch(kv8_append_kernel<kRopePairs>);
        case kRopeOddPairs: return launch(kv8_append_kernel<kRopeOddPairs>);
        default: return launch(kv8_append_kernel<kRopeOddHalves>);
    }
}
