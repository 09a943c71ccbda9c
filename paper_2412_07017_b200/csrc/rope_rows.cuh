// Rows of heads, turned by their tokens' positions and written as bf16 (rope.cu) or as rows of the 8-bit cache
// (kv8_append.cu).
//
// Rotary positions: pair j of a head's first rotary_dim values turns by the angle position * f_j,
//     (x, y) -> m (x cos a - y sin a, y cos a + x sin a),
// the pairs being (j, j + rotary_dim / 2) or (2j, 2j + 1), the others passing through.  The frequencies come as turns
// (f_j / 2 pi) in fp64, where position * turns is reduced to [-1/2, 1/2] and its sine and cosine are taken: an fp32
// angle is off by thousandths of a radian at positions of 10^5.  Both are kept as two fp32 numbers, a high part of 16
// bits, whose products with bf16 values are exact, and a low part, and a product difference x c - y s is evaluated from
// these (rope_diff): a value that is left over from two that cancel is as exact as any other down to 2^-18 of them, and
// is rounded once, to what is written.  That takes five fp32 instructions a value, without conversions to fp64, which
// run at an eighth of the rate of these.
//
// What bounds it: instructions and their latency more than memory (4097 tokens of 32 + 8 heads of 128 take 21.0 us, 4
// TB/s, with 62 % of the issue slots taken by two CTAs to an SM, which is what their registers leave room for) or, for
// few tokens, the latency of one chain: positions, angles, rows, stores (3.4 us in a graph).
// A thread holds 8 values of a row, 16 bytes; head_dim / 8 lanes hold a row, so a pair's other half comes by shuffle,
// and so does a row's maximum.  A warp takes kRopeUnroll times as many rows of ONE token as it has room for and
// requests them together: the sines and cosines of a lane's values are the same for all heads and are read from shared
// memory once.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "asynclm.h"
#include "common.cuh"
#include "kv8.cuh"

namespace asynclm {

constexpr int kRopeRowThreads = 256;
constexpr int kRopeUnroll = 4;
constexpr int kRopeMaxPairs = 128;
constexpr int kRopeEntries = kRopeMaxPairs + 8;      // of a token's table, see rope_entry

// Heads [T][heads][head_dim] of one tensor, rows `stride` values apart.
struct RowSet {
    const __nv_bfloat16* in;
    __nv_bfloat16* out;           // bf16 output, or null: a K or V set of the cache
    int64_t in_stride, out_stride;
    int32_t heads;
    int32_t turned;               // whether the rows are rotated
};

struct RopeTurns {
    double turns[kRopeMaxPairs];
    double factor;
    int32_t rotary_dim;           // 0: nothing turns
    int32_t layout;
};

// The kernels' forms: halves of whole 16-byte vectors, interleaved pairs that fill such vectors, halves that begin
// inside a vector, interleaved pairs that end inside one.  (Sorting the values of a cut vector where none is cut would
// cost the append of a prompt 3 %.)
enum RopeForm { kRopeHalves, kRopePairs, kRopeOddHalves, kRopeOddPairs };
constexpr bool rope_in_pairs(int form) { return form == kRopePairs || form == kRopeOddPairs; }
template <int FORM>
constexpr bool kInPairs = rope_in_pairs(FORM);
inline RopeForm rope_form(const RopeTurns& r) {
    if (r.layout == ASYNCLM_ROPE_INTERLEAVED) return r.rotary_dim % 8 == 0 ? kRopePairs : kRopeOddPairs;
    return r.rotary_dim % 16 == 0 ? kRopeHalves : kRopeOddHalves;
}
// CTAs of an SM and the most tokens of a CTA, by form.  The sines and cosines of a lane are 16 registers for pairs and
// 32 for halves, and rows in flight are worth more than registers for pairs only (8192 tokens of 32/8 heads, pairs,
// append: 54.5 us with two CTAs to an SM, 47.7 with three; 4097 tokens, halves: 23.3 with two and up to 8 tokens, 30.3
// with three, 21.2 with two and up to 16, where pairs take 56.9; all with one instruction a value more than now, 46.7
// and 21.0).
constexpr int rope_ctas(int form) { return rope_in_pairs(form) ? 3 : 2; }
constexpr int rope_most_tokens(int form) { return rope_in_pairs(form) ? 8 : 16; }
// Where pair j lies in a token's table: a lane reads `m` consecutive pairs, 8, 4 or each by itself, and lanes next to
// each other then read entries next to each other.
template <int FORM>
__device__ __forceinline__ constexpr int rope_group() { return kInPairs<FORM> ? 4 : FORM == kRopeHalves ? 8 : 1; }
__device__ __forceinline__ int rope_entry(int j, int m, int per) { return m == 1 ? j : (j % m) * per + j / m; }

// c as a high part of 16 bits and the rest, which has c's sign, and is not zero unless c is: see rope_diff.
__device__ __forceinline__ float2 rope_split(double c) {
    const float high = __uint_as_float(__float_as_uint(__double2float_rz(c)) & 0xffffff00u);
    const float low = (float)(c - (double)high);
    return make_float2(high, c != 0.0 && low == 0.f ? copysignf(1e-30f, high) : low);
}

// x c - y s with c = c.x + c.y, s = s.x + s.y, x and y bf16 numbers: their products with the high parts are exact, so
// the difference of these has one rounding, and the low parts are added last.  An infinite x or y makes the same
// infinity (or NaN) of both, because the parts have one sign: the sum is what the formula has.
__device__ __forceinline__ float rope_diff(float x, float2 c, float y, float2 s) {
    const float p = __fmul_rn(y, s.x);
    const float low = __fmaf_rn(x, c.y, -__fmul_rn(y, s.y));
    return __fadd_rn(__fmaf_rn(x, c.x, -p), low);
}

// Fills table[i][...] with m cos and m sin (high parts, then low parts) of tokens 0 .. n - 1 of the CTA.  A thread
// keeps one pair, whose frequency it reads from the kernel's parameters once (lanes that read different entries there
// take turns).
template <int FORM, typename Position>
__device__ __forceinline__ void rope_fill(const RopeTurns& r, float4 (*table)[kRopeEntries], int n, Position position) {
    const int pairs = r.rotary_dim / 2;
    if (pairs == 0) return;
    constexpr int m = rope_group<FORM>();
    const int per = (pairs + m - 1) / m;
    const int at_once = max(1, (int)blockDim.x / pairs);
    for (int a = threadIdx.x; a < at_once * pairs; a += blockDim.x) {      // (blocks of fewer threads than pairs: several pairs a thread)
        const int j = a % pairs;
        const double f = r.turns[j];
        const int e = rope_entry(j, m, per);
        for (int i = a / pairs; i < n; i += at_once) {
            const double t = (double)position(i) * f;
            double s, c;
            sincospi(2.0 * (t - rint(t)), &s, &c);
            c *= r.factor;
            s *= r.factor;
            const float2 cc = rope_split(c), ss = rope_split(s);
            table[i][e] = make_float4(cc.x, ss.x, cc.y, ss.y);
        }
    }
}

// This lane's sines and cosines: of its 8 values (halves), or of its 4 pairs (interleaved; c[k], s[k] for k < 4).
template <int FORM>
struct RopeLane { float2 c[kInPairs<FORM> ? 4 : 8], s[kInPairs<FORM> ? 4 : 8]; };

template <int FORM>
__device__ __forceinline__ RopeLane<FORM> rope_lane(const RopeTurns& r, const float4* table, int v) {
    RopeLane<FORM> x;
    constexpr int m = rope_group<FORM>();
    const int rd = r.rotary_dim, pairs = rd / 2, per = (pairs + m - 1) / m;
#pragma unroll
    for (int k = 0; k < (kInPairs<FORM> ? 4 : 8); ++k) {
        float4 cs = make_float4(1.f, 0.f, 0.f, 0.f);
        const int dim = 8 * v + k;
        if (kInPairs<FORM>) {
            if (4 * v + k < pairs) cs = table[k * per + v];
        } else if (dim < rd) {
            const bool second = dim >= pairs;
            const int j = second ? dim - pairs : dim;
            cs = table[rope_entry(j, m, per)];
            if (second) cs.y = -cs.y, cs.w = -cs.w;      // x c - y s for the first value of a pair, y c + x s for the second
        }
        x.c[k] = make_float2(cs.x, cs.z);
        x.s[k] = make_float2(cs.y, cs.w);
    }
    return x;
}

// y = the lane's 8 values of a row, turned.  All lanes of the warp take part.  `stage`: 512 bytes of the warp's own.
template <int FORM>
__device__ __forceinline__ void rope_turn(const RopeTurns& r, const RopeLane<FORM>& cs, int v, int lane, uint4* stage, const uint4& x, float (&y)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float own[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) { own[2 * k] = bf16_lo(w[k]); own[2 * k + 1] = bf16_hi(w[k]); }
    const int rd = r.rotary_dim, pairs = rd / 2;
    if constexpr (kInPairs<FORM>) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float a = own[2 * k], b = own[2 * k + 1];
            const bool on = 4 * v + (FORM == kRopePairs ? 0 : k) < pairs;      // (0 * infinity is not to reach a value that passes through)
            y[2 * k] = on ? rope_diff(a, cs.c[k], b, cs.s[k]) : a;
            y[2 * k + 1] = on ? rope_diff(b, cs.c[k], a, make_float2(-cs.s[k].x, -cs.s[k].y)) : b;
        }
    } else if constexpr (FORM == kRopeHalves) {
        // whole vectors: the pairs' other values are those of one other lane
        const int off = pairs / 8, other = v < off ? lane + off : v < 2 * off ? lane - off : lane;
        uint32_t p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = __shfl_sync(0xffffffffu, w[k], other);
        const bool on = v < 2 * off;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            y[2 * k] = on ? rope_diff(own[2 * k], cs.c[2 * k], bf16_lo(p[k]), cs.s[2 * k]) : own[2 * k];
            y[2 * k + 1] = on ? rope_diff(own[2 * k + 1], cs.c[2 * k + 1], bf16_hi(p[k]), cs.s[2 * k + 1]) : own[2 * k + 1];
        }
    } else {
        // halves that do not begin on a vector: through shared memory, value by value
        __syncwarp();
        stage[lane] = x;
        __syncwarp();
        const unsigned short* row = reinterpret_cast<const unsigned short*>(stage + (lane - v));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int dim = 8 * v + k;
            const float p = dim < rd ? __uint_as_float((uint32_t)row[dim < pairs ? dim + pairs : dim - pairs] << 16) : 0.f;
            y[k] = dim < rd ? rope_diff(own[k], cs.c[k], p, cs.s[k]) : own[k];
        }
    }
}

// The lane's 8 values as they are written: turned ones rounded, the others as they came, bit for bit (fp32 has no bf16
// NaN's payload and these kernels flush subnormal numbers). rotary_dim is even, so a word of two values is of one kind.
template <int FORM>
__device__ __forceinline__ uint4 rope_words(const RopeTurns& r, int v, const uint4& x, const float (&y)[8]) {
    const int left = r.rotary_dim - 8 * v;      // values of the lane that turn
    if (left <= 0) return x;
    uint4 o = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
    if (FORM == kRopeOddHalves || FORM == kRopeOddPairs) {
        if (left <= 2) o.y = x.y;
        if (left <= 4) o.z = x.z;
        if (left <= 6) o.w = x.w;
    }
    return o;
}

// Tokens of a CTA: one while that leaves SMs without a CTA; more are worked on beside each other.
inline int rope_row_tokens(int total, int form) {
    const int wave = 148 * (rope_in_pairs(form) ? 4 : 2), t = (total + wave - 1) / wave;
    return t < 1 ? 1 : t > rope_most_tokens(form) ? rope_most_tokens(form) : t;
}
// A warp's stage (512 bytes each) and the tables.
inline size_t rope_row_smem(int tokens) { return (size_t)kRopeRowThreads * sizeof(uint4) + (size_t)tokens * kRopeEntries * sizeof(float4); }

// The table's numbers as kernels take them; false if it is not one that asynclm_rope_table_init made for this head_dim.
bool rope_turns(const asynclm_rope_table* table, int head_dim, RopeTurns* out);

}  // namespace asynclm
