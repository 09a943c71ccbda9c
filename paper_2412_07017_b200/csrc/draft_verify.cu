// Drafted tokens held against the target's probabilities, and the token that follows the accepted ones.
//
// Draft i of a sequence, token x, is accepted if u_i q_i(x) < p_i(x) and all in front of it are; so a token is emitted with the target's probability
// whatever the draft proposed.  Behind the last accepted one, the next token has the weights w = max(p - q, 0) of the first rejected draft's row, or
// w = p of the row behind the last draft: the least t with sum_{t' <= t} w > u * sum w.
//
// The tests are products of two 24-bit numbers, and the search is for a place in a sum over the vocabulary whose steps may be 1e-7 of it: both are
// held in 64 bits, where neither depends on the order of the additions but within 2^-45.  A value becomes an fp64 one by its bits, without the
// exponents' difference in bias: all weights and sums are times 2^-896, which changes no comparison, and zeros and subnormal numbers are right as they
// are.  (With conversions, of which an SM does 16 a cycle, a mean batch of 300 bf16 rows of 100 003 took 45.7 us, 26.4 for 64 pairs of fp32 rows of 128 256.)
//
// One launch: a CTA takes a slice of one sequence's row (which row, every warp finds out for itself), a warp kPiece values of it at a time, and
// leaves each piece's sum in the workspace; the CTA that completes the row finds the piece by the sums, and reads that one again.  Every
// value is read once, so the bytes of one row of p and one of q a sequence are what bounds a large batch, and a chain of round trips (bounds of the
// sequence, tokens, their probabilities, values; count, sums, one piece) a small one.
#include <algorithm>

#include "asynclm.h"
#include "common.cuh"
#include "kernels.h"

namespace asynclm {

namespace {

constexpr int kVerifyThreads = 128, kVerifyWarps = kVerifyThreads / 32, kVerifyCtasPerSm = 8;
constexpr int kLaneValues = 16, kPiece = 32 * kLaneValues;
constexpr int kSharedPieces = 1024;
constexpr int kMostSequences = 65535;
constexpr size_t kArrivalBytes = 65536 * sizeof(int32_t);      // in front of the sums for any batch, so that calls of different sizes share a workspace

struct VerifyArgs {
    const int32_t* indptr;      // [batch + 1] over drafts
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    const int32_t* tokens;
    const float *accept_u, *sample_u;
    int32_t *accepted, *tokens_out;
    int32_t* arrivals;          // [batch], zero between launches
    double* sums;               // [batch][pieces]
    int32_t batch, drafts, vocab, pieces;
};

template <typename T>
struct Weights {
    const T *p, *q;      // q == nullptr: w = p
    int without;         // a token whose weight is zero (a draft proposed with certainty), or -1
    int vocab;
};

// The bits, as those of fp32 numbers, of the 16 bytes of values from `at` on of a row; zero behind its end.
template <typename T, bool VEC, int N>
__device__ __forceinline__ void load_values(const T* __restrict__ row, int at, int vocab, uint32_t (&x)[N]) {
    static_assert(N == 16 / sizeof(T), "a vector at a time");
    if (VEC && at + N <= vocab) {
        const uint4 w = ldg_nc_v4(reinterpret_cast<const uint4*>(row + at));
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (sizeof(T) == 4) x[i] = u[i];
            else x[i] = i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = at + i < vocab ? __float_as_uint((float)row[at + i]) : 0u;
}

// max(p - q, 0) times 2^-896, of fp32 numbers given by their bits.  NaN counts as zero, and so does a negative q.
__device__ __forceinline__ double scaled(uint32_t bits) { return __hiloint2double((int)(bits >> 3), (int)(bits << 29)); }
__device__ __forceinline__ double weight(uint32_t p, uint32_t q) {
    const uint32_t from = (uint32_t)max((int)q, 0);
    return __uint_as_float(p) > __uint_as_float(from) ? scaled(p) - scaled(from) : 0.0;
}
__device__ __forceinline__ double weight(uint32_t p) { return __uint_as_float(p) > 0.f ? scaled(p) : 0.0; }

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// Inclusive sums over the lanes.
__device__ __forceinline__ double warp_scan(double x, int lane) {
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    return x;
}

// The sums of pieces first, first + step, ... below `end` by this warp.
template <typename T, bool VEC, bool WITH_Q>
__device__ __forceinline__ void sum_pieces(const Weights<T>& w, int first, int step, int end, double* sums, int lane) {
    constexpr int N = 16 / sizeof(T), kParts = kLaneValues / N;
    for (int i = first; i < end; i += step) {
        uint32_t a[kParts][N], b[kParts][N];
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            const int at = i * kPiece + (k * 32 + lane) * N;
            load_values<T, VEC, N>(w.p, at, w.vocab, a[k]);
            if (WITH_Q) load_values<T, VEC, N>(w.q, at, w.vocab, b[k]);
        }
        if (!WITH_Q && w.without / kPiece == i) {      // (-1 / kPiece is 0)
#pragma unroll
            for (int k = 0; k < kParts; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (i * kPiece + (k * 32 + lane) * N + e == w.without) a[k][e] = 0;
        }
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < kParts; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) sum += WITH_Q ? weight(a[k][e], b[k][e]) : weight(a[k][e]);
        sum = warp_sum(sum);
        if (lane == 0) sums[i] = sum;
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void sum_pieces(const Weights<T>& w, int first, int step, int end, double* sums, int lane) {
    if (w.q != nullptr) sum_pieces<T, VEC, true>(w, first, step, end, sums, lane);
    else sum_pieces<T, VEC, false>(w, first, step, end, sums, lane);
}

// The least token whose inclusive sum of weights exceeds u * (sum of all); -1 if no weight is positive.  By one warp; sum_of(i): a piece's sum.
template <typename T, bool VEC, typename SumOf>
__device__ __forceinline__ int search(const Weights<T>& w, SumOf sum_of, int pieces, float u, int lane) {
    // a stretch of pieces to a lane, then the pieces of the stretch
    const int per = (pieces + 31) / 32, c0 = min(lane * per, pieces), c1 = min(c0 + per, pieces);
    double mine = 0.0;
    for (int c = c0; c < c1; ++c) mine += sum_of(c);
    const double upto = warp_scan(mine, lane), total = __shfl_sync(0xffffffffu, upto, 31);
    if (!(total > 0.0)) return -1;
    const double threshold = (double)u * total;
    // (Rounding may leave nothing beyond the threshold, and a u of one or more does: then the last with a weight.)
    const unsigned beyond = __ballot_sync(0xffffffffu, mine > 0.0 && upto > threshold), some = __ballot_sync(0xffffffffu, mine > 0.0);
    const int at = beyond ? __ffs(beyond) - 1 : 31 - __clz(some), at0 = at * per, at1 = min(at0 + per, pieces);
    double before = __shfl_sync(0xffffffffu, upto - mine, at);
    double front = before;
    int piece = at0;
    for (int c = at0; c < at1; c += 32) {
        const double x = c + lane < at1 ? sum_of(c + lane) : 0.0, through = before + warp_scan(x, lane);
        const unsigned past = __ballot_sync(0xffffffffu, x > 0.0 && through > threshold), any = __ballot_sync(0xffffffffu, x > 0.0);
        const double end = __shfl_sync(0xffffffffu, through, 31);
        if (any) {
            const int l = past ? __ffs(past) - 1 : 31 - __clz(any);
            piece = c + l;
            front = __shfl_sync(0xffffffffu, through - x, l);
        }
        if (past) break;
        before = end;
    }
    before = front;
    // the token: kLaneValues next to each other to a lane
    constexpr int N = 16 / sizeof(T);
    const int t0 = piece * kPiece + lane * kLaneValues;
    double x[kLaneValues], sum = 0.0;
#pragma unroll
    for (int k = 0; k < kLaneValues; k += N) {
        uint32_t a[N], b[N];
        load_values<T, VEC, N>(w.p, t0 + k, w.vocab, a);
        if (w.q != nullptr) load_values<T, VEC, N>(w.q, t0 + k, w.vocab, b);
#pragma unroll
        for (int e = 0; e < N; ++e) x[k + e] = t0 + k + e == w.without ? 0.0 : w.q != nullptr ? weight(a[e], b[e]) : weight(a[e]);
    }
#pragma unroll
    for (int k = 0; k < kLaneValues; ++k) sum += x[k];
    const double through = before + warp_scan(sum, lane);
    const unsigned past = __ballot_sync(0xffffffffu, sum > 0.0 && through > threshold), any = __ballot_sync(0xffffffffu, sum > 0.0);
    const int from = past ? __ffs(past) - 1 : 31 - __clz(any);
    int token = -1;
    double run = through - sum;
    bool found = false;
#pragma unroll
    for (int k = 0; k < kLaneValues; ++k) {
        run += x[k];
        if (!found && x[k] > 0.0) {
            token = t0 + k;
            found = run > threshold;
        }
    }
    return __shfl_sync(0xffffffffu, token, from);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kVerifyThreads, kVerifyCtasPerSm)
draft_verify_kernel(VerifyArgs a) {
    __shared__ int s_last, s_again;
    __shared__ double s_sums[kSharedPieces];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.y;
    pdl_wait();
    pdl_trigger();
    const int i0 = min(max(__ldg(a.indptr + b), 0), a.drafts), i1 = min(max(__ldg(a.indptr + b + 1), i0), a.drafts), n = i1 - i0;
    const T* target = reinterpret_cast<const T*>(a.target) + (int64_t)(i0 + b) * a.target_stride;
    const T* draft = a.draft == nullptr ? nullptr : reinterpret_cast<const T*>(a.draft) + (int64_t)i0 * a.draft_stride;
    // ---- how many are accepted: a draft to a lane
    int accepted = n, rejected_token = -1;
    for (int k0 = 0; k0 < n && accepted == n; k0 += 32) {
        const int k = k0 + lane;
        bool bad = false;
        int x = -1;
        if (k < n) {
            x = __ldg(a.tokens + i0 + k);
            bad = true;      // (a token outside the vocabulary has no probability)
            if (x >= 0 && x < a.vocab) {
                const double pv = (double)(float)target[(int64_t)k * a.target_stride + x];
                const double qv = draft == nullptr ? 1.0 : (double)(float)draft[(int64_t)k * a.draft_stride + x];
                bad = !((double)__ldg(a.accept_u + i0 + k) * qv < pv);
            }
        }
        const unsigned ballot = __ballot_sync(0xffffffffu, bad);
        if (ballot) {
            accepted = k0 + __ffs(ballot) - 1;
            rejected_token = __shfl_sync(0xffffffffu, x, __ffs(ballot) - 1);
        }
    }
    const bool rejected = accepted < n;
    Weights<T> w{target + (int64_t)accepted * a.target_stride, rejected && draft != nullptr ? draft + (int64_t)accepted * a.draft_stride : nullptr,
                 rejected && draft == nullptr ? rejected_token : -1, a.vocab};
    // ---- this CTA's slice of the row's pieces
    double* sums = a.sums + (size_t)b * a.pieces;
    const int first = (int)((int64_t)a.pieces * blockIdx.x / gridDim.x), end = (int)((int64_t)a.pieces * (blockIdx.x + 1) / gridDim.x);
    sum_pieces<T, VEC>(w, first + warp, kVerifyWarps, end, sums, lane);
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(a.arrivals + b, 1) == (int)gridDim.x - 1;
        if (s_last) {
            a.arrivals[b] = 0;      // ready for the next launch
            __threadfence();
        }
    }
    __syncthreads();
    if (!s_last) return;
    // ---- the CTA that completes the row
    const bool shared = a.pieces <= kSharedPieces;
    int token = -1;
    for (int attempt = 0; attempt < 2; ++attempt) {
        if (shared) {
            for (int i = threadIdx.x; i < a.pieces; i += kVerifyThreads) s_sums[i] = __ldcg(sums + i);
            __syncthreads();
        }
        if (warp == 0) {
            token = search<T, VEC>(w, [&](int i) { return shared ? s_sums[i] : __ldcg(sums + i); }, a.pieces, __ldg(a.sample_u + b), lane);
            if (lane == 0) s_again = token < 0 && rejected && attempt == 0;
        }
        __syncthreads();
        if (!s_again) break;
        // nothing is left of max(p - q, 0), as rounded probabilities may have it: the target's own
        w.q = nullptr;
        w.without = -1;
        sum_pieces<T, VEC>(w, warp, kVerifyWarps, a.pieces, sums, lane);
        __syncthreads();      // (the sums are this CTA's own now)
    }
    if (warp != 0) return;
    for (int k = lane; k <= n; k += 32) a.tokens_out[i0 + b + k] = k < accepted ? __ldg(a.tokens + i0 + k) : k == accepted ? token : -1;
    if (lane == 0) a.accepted[b] = accepted;
}

}  // namespace

}  // namespace asynclm

extern "C" size_t asynclm_draft_verify_workspace_bytes(int32_t batch, int32_t vocab) {
    using namespace asynclm;
    if (batch <= 0 || vocab <= 0) return 0;
    const size_t pieces = ((size_t)vocab + kPiece - 1) / kPiece;
    return kArrivalBytes + (size_t)batch * pieces * sizeof(double);
}

extern "C" int asynclm_draft_verify(const asynclm_draft_rows* rows, const int32_t* draft_indptr, int32_t batch, int32_t drafts, const int32_t* draft_tokens,
                                    const float* accept_u, const float* sample_u, int32_t* accepted, int32_t* tokens_out, void* workspace, void* stream) {
    using namespace asynclm;
    if (!rows || batch < 0 || drafts < 0 || rows->vocab <= 0 || rows->vocab > INT32_MAX - kPiece || batch > kMostSequences) return ASYNCLM_ERR_INVALID_ARG;
    if (rows->dtype != ASYNCLM_DTYPE_BF16 && rows->dtype != ASYNCLM_DTYPE_F32) return ASYNCLM_ERR_INVALID_ARG;
    if (batch == 0) return drafts == 0 ? ASYNCLM_OK : ASYNCLM_ERR_INVALID_ARG;
    if (!rows->target || !draft_indptr || !sample_u || !accepted || !tokens_out || !workspace || (drafts > 0 && (!draft_tokens || !accept_u)))
        return ASYNCLM_ERR_INVALID_ARG;
    if (rows->target_stride < rows->vocab || (rows->draft && rows->draft_stride < rows->vocab)) return ASYNCLM_ERR_INVALID_ARG;
    const uintptr_t size = rows->dtype == ASYNCLM_DTYPE_F32 ? 4 : 2;
    if ((((uintptr_t)rows->target | (uintptr_t)rows->draft) & (size - 1)) != 0 || ((uintptr_t)workspace & 15) != 0 ||
        (((uintptr_t)draft_indptr | (uintptr_t)draft_tokens | (uintptr_t)accept_u | (uintptr_t)sample_u | (uintptr_t)accepted | (uintptr_t)tokens_out) & 3) != 0)
        return ASYNCLM_ERR_INVALID_ARG;
    VerifyArgs a{};
    a.indptr = draft_indptr;
    a.target = rows->target;
    a.draft = rows->draft;
    a.target_stride = rows->target_stride;
    a.draft_stride = rows->draft ? rows->draft_stride : 0;
    a.tokens = draft_tokens;
    a.accept_u = accept_u;
    a.sample_u = sample_u;
    a.accepted = accepted;
    a.tokens_out = tokens_out;
    a.arrivals = (int32_t*)workspace;
    a.sums = (double*)((char*)workspace + kArrivalBytes);
    a.batch = batch;
    a.drafts = drafts;
    a.vocab = rows->vocab;
    a.pieces = (rows->vocab + kPiece - 1) / kPiece;
    // as many CTAs as run at once, each with a piece or more for its warps
    const int slices = std::max(1, std::min(kVerifyCtasPerSm * 148 / batch, (a.pieces + kVerifyWarps - 1) / kVerifyWarps));
    // rows that all start on a 16-byte boundary are read by vectors
    const bool vec = (((uintptr_t)a.target | (uintptr_t)a.draft | (uintptr_t)a.target_stride * size | (uintptr_t)a.draft_stride * size) & 15) == 0;
    auto kernel = size == 4 ? (vec ? draft_verify_kernel<float, true> : draft_verify_kernel<float, false>)
                            : (vec ? draft_verify_kernel<__nv_bfloat16, true> : draft_verify_kernel<__nv_bfloat16, false>);
    return cuda_status(launch_pdl(kernel, dim3(slices, batch), dim3(kVerifyThreads), 0, (cudaStream_t)stream, a));
}
