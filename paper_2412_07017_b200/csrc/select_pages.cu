// Which pages a token attends to: for every (token, kv head) the first and the last pages that it sees and, up to the budget, those whose keys
// could score highest.
//
// Score.  For a query q and a page whose keys lie between lo and hi, channel by channel, no key scores more than
//     sum_c max(q_c lo_c, q_c hi_c) = sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c;
// a page's score is the largest over the G queries of the kv head.  As two products it is a matrix product of bf16 operands, pages x queries.  But sums
// of 32 bits in different orders differ in their last bits, and with them the choice, wherever two pages are close; the choice shall depend on the
// values alone.  So it is made in two steps: scores from the tensor cores with a bound of their error, e = 2^-14 sum_c |q_c| max(|lo_c|, |hi_c|), the
// largest of the row; then, as the budget's last score t in 32 bits lies within e of the one in full, pages above t + 2e are in, pages below
// t - 2e are out, and the few in between (one to five, where scores are not equal) are scored again in 64 bits, where a product of bf16 values is exact.
//   (e: either product is D / 16 instructions one after the other, each of which adds 16 exact products to the sum; with truncation to 2^-23 of the largest
// for each of the 17 terms that is, over both, 16 * 17 * 2^-23 < 2^-14.9 of the sum of magnitudes for D = 128, and 2^-24 where they are added.  That the instruction does
// no worse is an assumption; the tests hold choices by products that cancel, with scores apart by 2^-6 to 2^-36 of a product, against 64 bits.)
//   In 64 bits for all pages the score kernel took 106 us for 48 sequences of 3-12 K tokens with 1-4 new ones each (451 K sums over 4 heads of 128):
// for every product a bit operation, an fma and a move, 112 instructions a sum; now it takes 22 us of 92 MB of bounds, and the choice 14.  (4 sequences of
// 16-60 K tokens: 13 us of 39 MB, and 7.)
//
// select_score_kernel: a warp takes 16 pages, the M of its MMAs, a CTA a stretch of a sequence's pages for one kv head and all of the sequence's rows
// (drafted tokens) at once.  Operands come from memory as they are: the k index may stand for any channel as long as it is the same for both
// sides, so a thread's 16 bytes of a page's row are two steps' fragments.  Bound by the bytes of the bounds.
// select_choose_kernel: a CTA for every (row, kv head).  A histogram of eight bits, from the first bit in which the scores differ, narrows t to one bin, whose
// keys are ranked against each other; then the pages in rising order, each thread a stretch of them.
#include <algorithm>

#include "asynclm.h"
#include "attn_launch.cuh"
#include "common.cuh"
#include "kernels.h"
#include "plan_internal.h"

namespace asynclm {

namespace {

constexpr int kScoreThreads = 128, kScoreWarps = kScoreThreads / 32;
constexpr int kTilePages = 16;
constexpr int kThreadKeys = 8;                     // of a row's keys in a thread's registers
constexpr unsigned kAlways = 0xffffffffu;          // key of a page that is taken whatever its score
constexpr unsigned kTaken = 0xfffffffeu;

// Values beyond +-2^56, NaN among them, count as +-2^56 (so that no sum of products overflows).
constexpr uint32_t kMostPair = 0x5b805b80u, kLeastPair = 0xdb80db80u, kAbs = 0x7fff7fffu;
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t held(uint32_t x) { return min2(max2(x, kLeastPair), kMostPair); }

__device__ __forceinline__ unsigned ordered(float x) {
    const unsigned u = __float_as_uint(x + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
// The page whose bounds are read for `id`, which the checked build holds against the pool's size.
__device__ __forceinline__ int bounds_page(const DevPlan& p, int id) { return page_ok(id, p.num_pages, p.status, kStatusBadPageSelect) ? id : 0; }

__device__ __forceinline__ float unordered(unsigned k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ unsigned long long ordered(double x) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// D (16x8, fp32) += A (16x16, bf16, row) . B (16x8, bf16, col)
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Of a warp: a tile of bounds in shared memory, [page][least, largest][channel], or two, one on its way while the other is in use, where that leaves room for
// as many CTAs as the registers do: at head_dim 128 five CTAs with a tile a warp do better than three with two (us of bounds, selection and
// attention 112.4 | 114.5 for 48 sequences, 36.8 | 37.7 for 4, at head_dim 64 43.2 | 42.5 for 150).  The 16-byte vectors of odd pages change places with
// those four further, so that the eight lanes that a bank serves at once (two pages, four vectors) read different ones.
template <int D>
struct ScoreSlots {
    static constexpr int kPageBytes = 4 * D, kBytes = kTilePages * kPageBytes, kSlots = D == 128 ? 1 : 2;
    static constexpr size_t kSmem = (size_t)kScoreWarps * kSlots * kBytes;
    static __device__ __forceinline__ int offset(int page, int vec) { return page * kPageBytes + (vec ^ (page & 1) * 4) * 16; }
};

// Thread (g, t) = (lane / 4, lane % 4) of an MMA holds channels 32 j + 8 t .. + 7 of pages g and g + 8 (A) and of query g (B): a 16-byte vector's
// first two words are the k columns 2t, 2t + 1 and 2t + 8, 2t + 9 of one instruction, its last two those of the next.
template <int D, int G>
__global__ void __launch_bounds__(kScoreThreads)
select_score_kernel(DevPlan p, const uint8_t* __restrict__ q, const uint8_t* __restrict__ bounds) {
    constexpr int J = D / 32, kColumns = 8, kGroups = kSelectQueries / kColumns;
    using Slots = ScoreSlots<D>;
    extern __shared__ __align__(16) uint8_t s_slots[];
    __shared__ uint4 s_q[kGroups][J][2][32];      // max(q, 0) and min(q, 0) as the threads take them
    __shared__ unsigned s_error[kSelectQueries];
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int h = blockIdx.x % p.num_kv_heads;
    const SelectChunk c = p.select_chunks[blockIdx.x / p.num_kv_heads];
    const int32_t* table = p.page_indices + c.page_base;
    const int pos0 = c.pos0;
    const int end = min(c.page0 + p.select_chunk_pages, (pos0 + c.rows - 1) / kPage + 1);
    const int queries = c.rows * G;
    auto id_of = [&](int j0) { return j0 + (lane & 15) < end ? bounds_page(p, __ldg(table + j0 + (lane & 15))) : -1; };
    constexpr int kStep = kScoreWarps * kTilePages;
    int j0 = c.page0 + warp * kTilePages, ids = id_of(j0), ids_next = id_of(j0 + kStep);
    // where this thread's scores go: of queries 2 t and, for one head to a row, 2 t + 1 of each eight
    constexpr int kMine = G == 1 ? 2 : 1;
    unsigned* keys[kGroups][kMine];
    int np[kGroups][kMine];      // pages that the row sees; 0: no such row, or another thread has it
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
#pragma unroll
        for (int e = 0; e < kMine; ++e) {
            const int query = k * kColumns + 2 * t + e, r = query / G;
            const bool on = query % G == 0 && r < c.rows;
            np[k][e] = on ? (pos0 + r) / kPage + 1 : 0;
            keys[k][e] = on ? p.select_keys + __ldg(p.select_base + c.row0 + r) * p.num_kv_heads + (size_t)h * np[k][e] : nullptr;
        }
    if (tid < kSelectQueries) s_error[tid] = 0;
    uint8_t* slots = s_slots + (size_t)warp * Slots::kSlots * Slots::kBytes;
    auto request = [&](int slot, int my_id) {
        constexpr int kVecs = Slots::kPageBytes / 16;      // of a page: all lanes, or half of them
#pragma unroll
        for (int i = 0; i < kTilePages * kVecs / 32; ++i) {
            const int page = (i * 32 + lane) / kVecs, vec = (i * 32 + lane) % kVecs;
            const int64_t id = __shfl_sync(0xffffffffu, my_id, page);
            const uint8_t* src = bounds + ((max(id, (int64_t)0) * p.num_kv_heads + h) * 2) * D * 2 + vec * 16;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(slots + slot * Slots::kBytes + Slots::offset(page, vec))),
                         "l"(src), "r"(id >= 0 ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    pdl_wait();      // queries and bounds are the kernels' in front
    // (all that is read first is on its way before any of it is waited for: a CTA's start takes longer than a tile)
    constexpr int kQueryVecs = kGroups * J * 32 / kScoreThreads;
    uint4 w[kQueryVecs];
#pragma unroll
    for (int n = 0; n < kQueryVecs; ++n) {
        const int i = tid + n * kScoreThreads, l = i % 32, j = i / 32 % J, k = i / 32 / J * kColumns + l / 4;
        w[n] = make_uint4(0, 0, 0, 0);
        if (k < queries)
            w[n] = *reinterpret_cast<const uint4*>(q + (((size_t)(c.row0 + k / G) * p.num_q_heads + (size_t)h * G + k % G) * D + 32 * j + 8 * (l % 4)) * 2);
    }
    if (j0 < end) request(0, ids);
#pragma unroll
    for (int n = 0; n < kQueryVecs; ++n) {
        const int i = tid + n * kScoreThreads;
        const uint4 x = make_uint4(held(w[n].x), held(w[n].y), held(w[n].z), held(w[n].w));
        s_q[i / 32 / J][i / 32 % J][0][i % 32] = make_uint4(max2(x.x, 0), max2(x.y, 0), max2(x.z, 0), max2(x.w, 0));
        s_q[i / 32 / J][i / 32 % J][1][i % 32] = make_uint4(min2(x.x, 0), min2(x.y, 0), min2(x.z, 0), min2(x.w, 0));
    }
    __syncthreads();
    float error[kGroups][2];
#pragma unroll
    for (int k = 0; k < kGroups; ++k) error[k][0] = error[k][1] = 0.f;
    for (int slot = 0; j0 < end; j0 += kStep) {
        const bool last = j0 + kStep >= end;
        const int next = Slots::kSlots == 2 ? slot ^ 1 : slot, ids_then = ids_next;
        if (Slots::kSlots == 2 && !last) {
            request(next, ids_then);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        ids_next = id_of(j0 + 2 * kStep);
        __syncwarp();      // all lanes' copies are there
        const uint8_t* tile = slots + slot * Slots::kBytes;
        const bool more = queries > kColumns;
        float s_all[kGroups][4], d_all[kGroups][4], a_all[kGroups][4];      // scores in two parts, sums of magnitudes
#pragma unroll
        for (int k = 0; k < kGroups; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_all[k][e] = d_all[k][e] = a_all[k][e] = 0.f;
#pragma unroll 1
        for (int j = 0; j < J; ++j) {      // (not unrolled: a launch's code is cold, and a CTA has one to four tiles a warp)
            uint32_t l[2][4], u[2][4], m[2][4];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint4 lo = *reinterpret_cast<const uint4*>(tile + Slots::offset(g + 8 * half, 4 * j + t));
                const uint4 hi = *reinterpret_cast<const uint4*>(tile + Slots::offset(g + 8 * half, D / 8 + 4 * j + t));
                const uint32_t x[4] = {lo.x, lo.y, lo.z, lo.w}, y[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    l[half][e] = held(x[e]);
                    u[half][e] = held(y[e]);
                    m[half][e] = max2(l[half][e] & kAbs, u[half][e] & kAbs);
                }
            }
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                if (k > 0 && !more) break;
                const uint4 up = s_q[k][j][0][lane], down = s_q[k][j][1][lane];
                float(&s)[4] = s_all[k], (&d)[4] = d_all[k], (&a)[4] = a_all[k];
                mma16(s, u[0][0], u[1][0], u[0][1], u[1][1], up.x, up.y);
                mma16(s, u[0][2], u[1][2], u[0][3], u[1][3], up.z, up.w);
                mma16(d, l[0][0], l[1][0], l[0][1], l[1][1], down.x, down.y);
                mma16(d, l[0][2], l[1][2], l[0][3], l[1][3], down.z, down.w);
                mma16(a, m[0][0], m[1][0], m[0][1], m[1][1], (up.x | down.x) & kAbs, (up.y | down.y) & kAbs);
                mma16(a, m[0][2], m[1][2], m[0][3], m[1][3], (up.z | down.z) & kAbs, (up.w | down.w) & kAbs);
            }
        }
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            if (k > 0 && !more) break;
            float(&s)[4] = s_all[k];
            const float(&a)[4] = a_all[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += d_all[k][e];
            // this thread: pages g (0, 1) and g + 8 (2, 3), queries 2 t and 2 t + 1 of the eight
            error[k][0] = fmaxf(error[k][0], fmaxf(a[0], a[2]));
            error[k][1] = fmaxf(error[k][1], fmaxf(a[1], a[3]));
            // the largest over a row's heads
            if constexpr (G >= 2) {
                s[0] = fmaxf(s[0], s[1]);
                s[2] = fmaxf(s[2], s[3]);
#pragma unroll
                for (int off = 1; off < G / 2; off <<= 1) {
                    s[0] = fmaxf(s[0], __shfl_xor_sync(0xffffffffu, s[0], off));
                    s[2] = fmaxf(s[2], __shfl_xor_sync(0xffffffffu, s[2], off));
                }
            }
#pragma unroll
            for (int e = 0; e < kMine; ++e)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int j = j0 + g + 8 * half;
                    if (j < min(end, np[k][e])) keys[k][e][j] = j < p.select_first || j >= np[k][e] - p.select_last ? kAlways : ordered(s[2 * half + e]);
                }
        }
        __syncwarp();      // (the slot is free)
        if (Slots::kSlots == 1 && !last) request(next, ids_then);
        slot = next;
    }
    // ---- how far the scores may be off: a row's largest (positive floats compare as integers)
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x = error[k][e];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
            if (g == 0) atomicMax(&s_error[k * kColumns + 2 * t + e], __float_as_uint(x));
        }
    __syncthreads();
    if (tid < queries) atomicMax(p.select_error + (size_t)(c.row0 + tid / G) * p.num_kv_heads + h, s_error[tid]);
}

// A bf16 number as held() has it, exactly (fp32 instructions would flush subnormal ones): the exponent field goes into an fp64 number's, whose bias is
// 896 more.
__device__ __forceinline__ double held_value(__nv_bfloat16 x) {
    const uint32_t bits = __bfloat16_as_ushort(x);
    if ((bits & 0x7fffu) > 0x7f80u) return -0x1p56;
    const int32_t word = ((int32_t)(bits << 16) >> 3) & (int32_t)0x8fffe000;
    return fmin(fmax(__hiloint2double(word, 0) * 0x1p896, -0x1p56), 0x1p56);
}

// The sum of one query in shared memory and a page's bounds in 64 bits, by a warp.
__device__ __forceinline__ double exact_sum(const __nv_bfloat16* q, const __nv_bfloat16* __restrict__ bounds, int head_dim, int lane) {
    const int n = head_dim / 32, at = n * lane;      // four channels to a lane, or two
    __nv_bfloat162 l[2], u[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l[i] = reinterpret_cast<const __nv_bfloat162*>(bounds + at)[n == 4 ? i : 0];
        u[i] = reinterpret_cast<const __nv_bfloat162*>(bounds + head_dim + at)[n == 4 ? i : 0];
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (2 * i >= n) break;
        const double x = held_value(q[at + 2 * i]), y = held_value(q[at + 2 * i + 1]);
        s = fma(x, held_value(x < 0.0 ? l[i].x : u[i].x), s);
        s = fma(y, held_value(y < 0.0 ? l[i].y : u[i].y), s);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    return s;
}

// A warp has the keys of a stretch of pages, 32 of them at a time, in registers where the row has at most kThreadKeys for every thread.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
select_choose_kernel(DevPlan p, const __nv_bfloat16* __restrict__ q, const __nv_bfloat16* __restrict__ bounds, int32_t* __restrict__ pages_out) {
    constexpr int kWarps = THREADS / 32;
    __shared__ unsigned s_some[THREADS];               // the keys of t's bin; the pages that are scored again,
    __shared__ int s_ids[THREADS];                     // and where they are
    __shared__ unsigned long long s_exact[THREADS];
    __shared__ int s_hist[256];
    __shared__ unsigned s_lo[kWarps], s_hi[kWarps], s_threshold;
    __shared__ int s_count[kWarps][2];
    __shared__ int s_bin, s_above, s_in, s_n, s_open, s_total;
    __shared__ __align__(16) __nv_bfloat16 s_q[8 * 128];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / p.num_kv_heads, h = blockIdx.x % p.num_kv_heads, seq = __ldg(p.row_seq + row);
    const size_t row_keys = (size_t)__ldg(p.select_base + row) * p.num_kv_heads;
    const int np = (__ldg(p.kv_len_before + seq) + row - __ldg(p.q_indptr + seq)) / kPage + 1;      // pages that the row sees
    const int32_t* table = p.page_indices + __ldg(p.page_indptr + seq);
    const int budget = p.select_budget;
    int32_t* list = p.select_pages + (size_t)blockIdx.x * budget;
    int32_t* out = pages_out == nullptr ? nullptr : pages_out + (size_t)blockIdx.x * budget;
    unsigned* keys = p.select_keys + row_keys + (size_t)h * np;
    const int steps = (np + THREADS - 1) / THREADS, stretch0 = warp * steps * 32;
    const bool resident = steps <= kThreadKeys;
    unsigned mine[kThreadKeys];
    int ids[kThreadKeys];
#pragma unroll
    for (int i = 0; i < kThreadKeys; ++i) {
        const int j = stretch0 + 32 * i + lane;
        ids[i] = resident && i < steps && j < np ? __ldg(table + j) : 0;
    }
    for (int i = tid; i < 256; i += THREADS) s_hist[i] = 0;
    if (tid == 0) s_n = s_open = s_total = 0;
    pdl_trigger();
    pdl_wait();      // the scores; and the lists belong to the last attention as long as it runs
    if (np <= budget) {
        for (int j = tid; j < budget; j += THREADS) {
            if (j < np) list[j] = __ldg(table + j);
            if (out != nullptr) out[j] = j < np ? j : -1;
        }
        return;
    }
    // ---- this thread's keys: pages stretch0 + 32 i + lane
#pragma unroll
    for (int i = 0; i < kThreadKeys; ++i) {
        const int j = stretch0 + 32 * i + lane;
        mine[i] = resident && i < steps && j < np ? __ldcg(keys + j) : 0;      // (0 is below any score's)
    }
    const float error = __uint_as_float(__ldcg(p.select_error + blockIdx.x)) * 0x1p-14f + 0x1p-60f;      // (products with subnormal numbers may be lost)
    const int D = p.head_dim, G = p.group;
    for (int i = tid; i < G * D / 8; i += THREADS)
        reinterpret_cast<uint4*>(s_q)[i] = reinterpret_cast<const uint4*>(q + ((size_t)row * p.num_q_heads + (size_t)h * G) * D)[i];
    // use(page, key, id) for each of them, all lanes together; use returns the key, or another to put in its place
    auto each = [&](auto use) {
        if (resident) {
#pragma unroll
            for (int i = 0; i < kThreadKeys; ++i)
                if (i < steps) mine[i] = use(stretch0 + 32 * i + lane, mine[i], ids[i]);
        } else {
            for (int i = 0; i < steps; ++i) {
                const int j = stretch0 + 32 * i + lane;
                const unsigned k = j < np ? __ldcg(keys + j) : 0, now = use(j, k, j < np ? __ldg(table + j) : 0);
                if (now != k && j < np) __stcg(keys + j, now);
            }
        }
    };
    unsigned lo = ~0u, hi = 0;      // of the scores
    each([&](int, unsigned k, int) {
        if (k != kAlways && k != 0) lo = min(lo, k), hi = max(hi, k);
        return k;
    });
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) s_lo[warp] = lo, s_hi[warp] = hi;
    __syncthreads();
    if (tid == 0) p.select_error[blockIdx.x] = 0;      // (all have read it) ready for the next launch
#pragma unroll
    for (int w = 0; w < kWarps; ++w) lo = min(lo, s_lo[w]), hi = max(hi, s_hi[w]);
    // ---- t: the need-th largest of the scores
    int need = budget - p.select_first - p.select_last;
    if (need == 0) {
        lo = kAlways, hi = kAlways - 1;
    } else {
        const int all = need;
        int shift = lo == hi ? 0 : max(0, 24 - __clz(lo ^ hi));
        while (true) {
            const unsigned base = lo >> shift;
            each([&](int, unsigned k, int) {
                if (k >= lo && k <= hi) atomicAdd(&s_hist[(k >> shift) - base], 1);
                return k;
            });
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
                    int bin = 0, in = 0;
#pragma unroll
                    for (int i = 7; i >= 0; --i)      // (from the highest: the first with which `need` is reached)
                        if (in == 0) {
                            if (above + n[i] >= need) bin = 8 * lane + i, in = n[i];
                            else above += n[i];
                        }
                    s_bin = bin;
                    s_above = above;
                    s_in = in;
                }
            }
            __syncthreads();
            const int in = s_in;
            need -= s_above;
            const unsigned first = (base + (unsigned)s_bin) << shift, last = first + ((1u << shift) - 1);
            lo = max(lo, first);
            hi = min(hi, last);
            if (shift == 0) break;
            if (in <= THREADS) {      // few: the need-th of them by rank
                each([&](int, unsigned k, int) {
                    if (k >= lo && k <= hi) s_some[atomicAdd(&s_n, 1)] = k;
                    return k;
                });
                __syncthreads();
                if (tid < in) {
                    const unsigned k = s_some[tid];
                    int above = 0, equal = 0;
                    for (int i = 0; i < in; ++i) above += s_some[i] > k, equal += s_some[i] == k;
                    if (above < need && need <= above + equal) s_threshold = k;      // (the same from all equal ones)
                }
                __syncthreads();
                lo = s_threshold;
                break;
            }
            shift = max(0, shift - 8);
            for (int i = tid; i < 256; i += THREADS) s_hist[i] = 0;
            __syncthreads();
        }
        // ---- scores within 2 e of it decide nothing
        const float t = unordered(lo);
        lo = ordered(__fadd_rd(t, -2.f * error));
        hi = ordered(__fadd_ru(t, 2.f * error));
        int above = 0;
        each([&](int j, unsigned k, int id) {
            above += k > hi && k != kAlways;
            if (k >= lo && k <= hi) {
                const int at = atomicAdd(&s_open, 1);
                if (at < THREADS) s_some[at] = (unsigned)j, s_ids[at] = id;
            }
            return k;
        });
        above = __reduce_add_sync(0xffffffffu, above);
        if (lane == 0) atomicAdd(&s_total, above);
        __syncthreads();
        need = all - s_total;      // to be taken of these
        const int open = s_open;
        if (open > need) {
            auto exact = [&](int id, int g) { return ordered(exact_sum(s_q + g * D, bounds + (((size_t)bounds_page(p, id) * p.num_kv_heads + h) * 2) * D, D, lane)); };
            if (open <= THREADS) {
                s_exact[tid] = 0;
                __syncthreads();
#pragma unroll 1
                for (int i = warp; i < open * G; i += kWarps) {      // a page and head to a warp: the code is met once, and cold
                    const unsigned long long x = exact(s_ids[i / G], i % G);
                    if (lane == 0) atomicMax(&s_exact[i / G], x);
                }
                __syncthreads();
                // an open page is in if fewer than `need` go in front of it (of equal scores the lower page)
                each([&](int j, unsigned k, int id) {
                    if (k < lo || k > hi) return k;
                    unsigned long long x = 0;
                    for (int i = 0; i < open; ++i)
                        if (s_some[i] == (unsigned)j) x = s_exact[i];
                    int rank = 0;
                    for (int i = 0; i < open; ++i) rank += s_exact[i] > x || (s_exact[i] == x && s_some[i] < (unsigned)j);
                    return rank < need ? kTaken : 0u;
                });
                need = 0;
            } else {
                // many scores that are (nearly) equal: the least of those in, bit by bit
                unsigned long long* all_exact = p.select_exact + row_keys + (size_t)h * np;
                each([&](int j, unsigned k, int id) {
                    unsigned which = __ballot_sync(0xffffffffu, k >= lo && k <= hi);
                    for (; which; which &= which - 1) {
                        const int at = __shfl_sync(0xffffffffu, j, __ffs(which) - 1), page = __shfl_sync(0xffffffffu, id, __ffs(which) - 1);
                        unsigned long long x = 0;
                        for (int g = 0; g < G; ++g) x = max(x, exact(page, g));
                        if (lane == 0) __stcg(all_exact + at, x);
                    }
                    return k;
                });
                auto count = [&](unsigned long long least) {      // of the open ones, with at least this
                    __syncthreads();
                    if (tid == 0) s_total = 0;
                    __syncthreads();
                    int n = 0;
                    each([&](int j, unsigned k, int id) {
                        if (k >= lo && k <= hi) n += __ldcg(all_exact + j) >= least;
                        return k;
                    });
                    n = __reduce_add_sync(0xffffffffu, n);
                    if (lane == 0) atomicAdd(&s_total, n);
                    __syncthreads();
                    return s_total;
                };
                unsigned long long least = 0;
                for (int bit = 63; bit >= 0; --bit)
                    if (count(least | 1ull << bit) >= need) least |= 1ull << bit;
                need -= count(least + 1);      // (no score is the largest integer)
                each([&](int j, unsigned k, int id) {
                    if (k < lo || k > hi) return k;
                    const unsigned long long x = __ldcg(all_exact + j);
                    return x > least ? kTaken : x == least ? hi : 0u;
                });
                lo = hi;
            }
        }
    }
    // ---- the list: pages with keys above `hi`, and the first `need` of those from `lo` to `hi`
    int above = 0, among = 0;      // of the warp's stretch
    each([&](int, unsigned k, int) {
        above += __popc(__ballot_sync(0xffffffffu, k > hi));
        among += __popc(__ballot_sync(0xffffffffu, k >= lo && k <= hi));
        return k;
    });
    if (lane == 0) s_count[warp][0] = above, s_count[warp][1] = among;
    __syncthreads();
    above = among = 0;      // in front of the stretch
    for (int w = 0; w < warp; ++w) above += s_count[w][0], among += s_count[w][1];
    const unsigned below = (1u << lane) - 1;
    each([&](int j, unsigned k, int id) {
        const unsigned over = __ballot_sync(0xffffffffu, k > hi), in = __ballot_sync(0xffffffffu, k >= lo && k <= hi);
        const int among_here = among + __popc(in & below);
        if (k > hi || (k >= lo && k <= hi && among_here < need)) {
            const int at = above + __popc(over & below) + min(among_here, need);
            list[at] = id;
            if (out != nullptr) out[at] = j;
        }
        above += __popc(over);
        among += __popc(in);
        return k;
    });
}

template <int D, int G>
cudaError_t launch_scores(const DevPlan& p, const void* q, const void* bounds, cudaStream_t s) {
    constexpr size_t smem = ScoreSlots<D>::kSmem;
    if (cudaError_t e = allow_smem<select_score_kernel<D, G>>(smem)) return e;
    return launch_when(!p.full_launch, select_score_kernel<D, G>, dim3((unsigned)(p.num_select_chunks * p.num_kv_heads)), dim3(kScoreThreads), smem, s, p,
                      (const uint8_t*)q, (const uint8_t*)bounds);
}

// As many threads as hold the longest row's keys in registers, 128 to 512: a short row's steps are fewer barriers than work.
cudaError_t launch_choice(const DevPlan& p, const void* q, const void* bounds, int32_t* pages_out, cudaStream_t s) {
    const dim3 grid((unsigned)(p.total_q * p.num_kv_heads));
    auto run = [&](auto kernel, int threads) {
        return launch_when(!p.full_launch, kernel, grid, dim3(threads), 0, s, p, (const __nv_bfloat16*)q, (const __nv_bfloat16*)bounds, pages_out);
    };
    if (p.select_most_pages <= 128 * kThreadKeys) return run(select_choose_kernel<128>, 128);
    if (p.select_most_pages <= 256 * kThreadKeys) return run(select_choose_kernel<256>, 256);
    return run(select_choose_kernel<512>, 512);
}

template <int D>
int select_d(PlanUse& use, const void* q, const void* bounds, int32_t* pages_out, cudaStream_t s) {
    if (use.dev.num_select_chunks > 0) {
        auto scores = use.dev.group == 1 ? launch_scores<D, 1> : use.dev.group == 2 ? launch_scores<D, 2> : use.dev.group == 4 ? launch_scores<D, 4>
                                                                                                                         : launch_scores<D, 8>;
        if (int rc = cuda_status(use.launched(scores(use.dev, q, bounds, s)))) return rc;
    }
    return cuda_status(use.launched(launch_choice(use.dev, q, bounds, pages_out, s)));
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
    const int rc = use.dev.head_dim == 128 ? select_d<128>(use, q, key_bounds, pages_out, s) : select_d<64>(use, q, key_bounds, pages_out, s);
    if (rc == ASYNCLM_OK) __atomic_store_n(&plan->selected, 1, __ATOMIC_RELEASE);
    return rc;
}
