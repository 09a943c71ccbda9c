// Drafted tokens held against the target's probabilities, and the token that follows the accepted ones.
//
// Draft i of a sequence, token x, is accepted if u_i q_i(x) < p_i(x) and all in front of it are; so a token is emitted with the target's probability
// whatever the draft proposed.  Behind the last accepted one, the next token has the weights w = max(p - q, 0) of the first rejected draft's row, or
// w = p of the row behind the last draft: the least t with sum_{t' <= t} w > u * sum w.
//
// The tests are products of two 24-bit numbers, and the search is for a place in a sum over the vocabulary whose steps may be 1e-7 of it: both are
// held in 64 bits, where neither depends on the order of the additions but within 2^-45.  A value becomes an fp64 one by its bits, without the
// exponents' difference in bias: all weights and sums are times 2^-896, which changes no comparison, and zeros and subnormal numbers are right as they
// are.  (With conversions, of which an SM does 16 a cycle, 300 bf16 rows of 100 003 took 45.7 us and 64 pairs of fp32 rows of 128 256 26.4; now, in a graph
// with inputs in cache, 18.9 and 16.6, out of cache 20.3 and 19.3, 3.0 and 3.1 TB/s; two sequences of four drafts from 32 001 tokens 7.4.)
//
// One launch: a CTA takes a slice of one sequence's row (which row, every warp finds out for itself); a warp has pieces of 2 KB brought into shared memory, the
// next one while it sums the last, and leaves each piece's sum in the workspace; the CTA that completes the row finds the piece by the sums, and brings
// that one again.  (Where nothing is left of max(p - q, 0), that CTA sums all of p's row by itself.)  Every value is read once, so the bytes of one row of p and one of q a sequence are what bounds a large batch, and a chain of
// round trips (bounds of the sequence, tokens, their probabilities, values; count, sums, one piece) a small one.  Rows start anywhere: what is copied are
// the 16-byte vectors that memory has them in, and shared memory is read by vectors, or value by value where q's do not lie as p's.  How many CTAs a row has: draft_grid.h.  (Out of registers, by vectors, with the checks that the ends of
// a row need, the loop outgrew the instruction cache or the registers: 300 bf16 rows of 100 003 took 33 to 126 us.)
#include <algorithm>
#include <atomic>

#include "asynclm.h"
#include "common.cuh"
#include "draft_grid.h"
#include "kernels.h"

namespace asynclm {

namespace {

constexpr int kPieceBytes = 2048;
template <typename T>
constexpr int kPiece = kPieceBytes / (int)sizeof(T);
constexpr int kSlots = 2;      // of a warp: a piece of p, and one of q with a vector more
constexpr int kSlotBytes = kPieceBytes, kSlotBytesQ = 2 * kPieceBytes + 16;
constexpr int kSharedPieces = kSlots * kSlotBytes / 8;
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

// The rows that a token's weight comes from.  A piece is so many values of p from a 16-byte boundary on; the first begins `lead` values in front of
// the row.  q's values lie `apart` values further behind a boundary of theirs.
template <typename T>
struct Weights {
    static constexpr int N = 16 / sizeof(T);
    const T *p, *q;      // q == nullptr: w = p
    int without;         // a token whose weight is zero (a draft proposed with certainty), or -1
    int vocab;
    int lead, apart;

    __device__ __forceinline__ Weights(const T* p_, const T* q_, int without_, int vocab_)
        : p(p_), q(q_), without(without_), vocab(vocab_), lead((int)((uintptr_t)p_ % 16 / sizeof(T))),
          apart((int)(((uintptr_t)q_ / sizeof(T) - (uintptr_t)p_ / sizeof(T)) % N)) {}

    __device__ __forceinline__ int token0(int piece) const { return piece * kPiece<T> - lead; }
};

__device__ __forceinline__ void copy_vec(uint32_t dst, uintptr_t src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// Requests a piece of a row, the first vector of which begins at value `from` (a boundary), and `more` vectors behind it into dst; zeros behind the row's
// end.  (The first vector may begin in front of the row: what is read there lies in the 16 bytes of the row's first value.)
template <typename T>
__device__ __forceinline__ void request(T* dst, const T* row, int from, int more, int vocab, int lane) {
    constexpr int N = 16 / sizeof(T), kVecs = kPieceBytes / 16;
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst) + 16 * lane;
    if (from >= 0 && from + (kVecs + more) * N <= vocab) {
        const uintptr_t src = (uintptr_t)(row + from) + 16 * lane;
#pragma unroll
        for (int k = 0; k < kVecs; k += 32) copy_vec(to + 16 * k, src + 16 * k, 16);
        if (lane < more) copy_vec(to + 16 * kVecs, src + 16 * kVecs, 16);
        return;
    }
#pragma unroll 1
    for (int k = 0; k < kVecs + more; k += 32) {
        const int at = from + (k + lane) * N, bytes = at + N <= 0 ? 0 : max(min(vocab - at, N), 0) * (int)sizeof(T);
        if (k + lane < kVecs + more) copy_vec(to + 16 * k, (uintptr_t)(row + (bytes > 0 ? at : 0)) & ~(uintptr_t)15, bytes);      // (of no bytes: any address)
    }
}
template <typename T>
__device__ __forceinline__ void request_piece(const Weights<T>& w, T* slot, int piece, int lane) {
    request(slot, w.p, w.token0(piece), 0, w.vocab, lane);
    if (w.q != nullptr) request(slot + kPiece<T>, w.q, w.token0(piece) - w.apart, w.apart ? 1 : 0, w.vocab, lane);
}
// What has come of a piece is made fit to be summed: nothing in front of the row, no weight for `without`.
template <typename T>
__device__ __forceinline__ void clean_piece(const Weights<T>& w, T* slot, int piece, int lane) {
    __syncwarp();      // (all lanes' copies are there)
    if (piece == 0 && lane < w.lead) slot[lane] = (T)0.f;
    const int at = w.without - w.token0(piece);
    if (w.without >= 0 && at >= 0 && at < kPiece<T> && lane == 0) slot[at] = (T)0.f;
    __syncwarp();
}
__device__ __forceinline__ uint32_t bits_of(float x) { return __float_as_uint(x); }
__device__ __forceinline__ uint32_t bits_of(__nv_bfloat16 x) { return (uint32_t)__bfloat16_as_ushort(x) << 16; }

// (The compiler's comparisons and conversions of fp32 numbers flush subnormal ones, and a sum that has what a comparison does not see would send the search
// to a place without a weight.  So all of it goes by the bits.)
//
// A positive number times 2^-896.
__device__ __forceinline__ double scaled(uint32_t bits) { return __hiloint2double((int)(bits >> 3), (int)(bits << 29)); }
// The number for the test of acceptance: a negative one counts as zero, NaN of either sign stays.
__device__ __forceinline__ double probability(uint32_t bits) {
    if ((int)bits < 0 && bits <= 0xff800000u) return 0.0;
    return bits & 0x7f800000u ? (double)__uint_as_float(bits) : scaled(bits) * 0x1p896;
}

// max(p - q, 0) times 2^-896, of fp32 numbers given by their bits.  Where p or q is NaN, of either sign, there is no weight; a negative q counts as zero.
template <bool WITH_Q>
__device__ __forceinline__ double weight(uint32_t p, uint32_t q) {
    if constexpr (!WITH_Q) return p - 1 < 0x7f800000u ? scaled(p) : 0.0;
    const uint32_t from = q - 0x80000000u <= 0x7f800000u ? 0u : q;      // (what is left with a sign is NaN, and greater than any p)
    const double left = scaled(p) - scaled(from);
    return p > from && p <= 0x7f800000u ? left : 0.0;
}
// The weight of value j of a piece in its slot.
template <typename T>
__device__ __forceinline__ double weight_in(const Weights<T>& w, const T* slot, int j) {
    return w.q != nullptr ? weight<true>(bits_of(slot[j]), bits_of(slot[kPiece<T> + w.apart + j])) : weight<false>(bits_of(slot[j]), 0u);
}

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

// The sum of a piece in its slot, lane by lane: value by value, whatever the numbers and q's place.  (Hardly ever met: kept short.)
template <typename T, bool WITH_Q>
__device__ __forceinline__ double sum_of_any(const T* slot, int apart, int lane) {
    double sum = 0.0;
#pragma unroll 1
    for (int j = lane; j < kPiece<T>; j += 32) sum += weight<WITH_Q>(bits_of(slot[j]), WITH_Q ? bits_of(slot[kPiece<T> + apart + j]) : 0u);
    return sum;
}
// The same of probabilities; `odd` is set where a number is none, and the sum is none then.  (Bits compare as the numbers do where no sign is set and p is no NaN.  A
// NaN among p that is greater than q adds 2^104 or more, the step of the numbers in front of infinity.)
constexpr double kOddSum = 0x1p-792;      // 2^104 times 2^-896
template <typename T>
__device__ __forceinline__ double sum_by_values(const T* slot, int apart, int lane, bool& odd) {
    double sum = 0.0;
    uint32_t signs = 0;
#pragma unroll 4
    for (int j = lane; j < kPiece<T>; j += 32) {
        const uint32_t a = bits_of(slot[j]), b = bits_of(slot[kPiece<T> + apart + j]);
        signs |= a | b;
        if (a > b) sum += scaled(a) - scaled(b);
    }
    odd = signs >> 31 || sum >= kOddSum;
    return sum;
}
// The same by vectors, where q's lie as p's do, or without q.
template <typename T, bool WITH_Q>
__device__ __forceinline__ double sum_by_vectors(const T* slot, int lane, bool& odd) {
    constexpr int N = 16 / sizeof(T);
    double sum[2] = {0.0, 0.0};
    uint32_t signs = 0, most = 0;
#pragma unroll 4
    for (int k = lane; k < kPieceBytes / 16; k += 32) {
        const uint4 v = reinterpret_cast<const uint4*>(slot)[k];
        const uint4 u = WITH_Q ? reinterpret_cast<const uint4*>(slot + kPiece<T>)[k] : make_uint4(0, 0, 0, 0);
        const uint32_t x[4] = {v.x, v.y, v.z, v.w}, y[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (!WITH_Q) most = sizeof(T) == 4 ? max(most, x[i]) : __vmaxu2(most, x[i]);
            else signs |= x[i] | y[i];
#pragma unroll
            for (int e = 0; e < N / 4; ++e) {
                const uint32_t a = sizeof(T) == 4 ? x[i] : e ? x[i] & 0xffff0000u : x[i] << 16, b = sizeof(T) == 4 ? y[i] : e ? y[i] & 0xffff0000u : y[i] << 16;
                if constexpr (!WITH_Q) sum[i & 1] += scaled(a);
                else if (a > b) sum[i & 1] += scaled(a) - scaled(b);
            }
        }
    }
    const double all = sum[0] + sum[1];
    if constexpr (WITH_Q) odd = (signs & (sizeof(T) == 4 ? 0x80000000u : 0x80008000u)) != 0 || all >= kOddSum;
    else if constexpr (sizeof(T) == 4) odd = most > 0x7f800000u;
    else odd = most >> 16 > 0x7f80u || (most & 0xffffu) > 0x7f80u;
    return all;
}
template <typename T, bool WITH_Q>
__device__ __forceinline__ double sum_of_piece(const T* slot, int apart, int lane) {
    bool odd;
    double sum;
    if (!WITH_Q || apart == 0) sum = sum_by_vectors<T, WITH_Q>(slot, lane, odd);
    else sum = sum_by_values(slot, apart, lane, odd);
    return __any_sync(0xffffffffu, odd) ? sum_of_any<T, WITH_Q>(slot, apart, lane) : sum;
}

// The sums of pieces first, first + step, ... below `end` by this warp, in its two slots.
template <typename T>
__device__ __forceinline__ void sum_pieces(const Weights<T>& w, T* slots, int slot_values, int first, int step, int end, double* sums, int lane) {
    auto ask = [&](int i, int slot) {
        if (i < end) request_piece(w, slots + slot * slot_values, i, lane);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    ask(first, 0);
    int at = 0;
    for (int i = first; i < end; i += step, at ^= 1) {
        ask(i + step, at ^ 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        T* slot = slots + at * slot_values;
        clean_piece(w, slot, i, lane);
        const double sum = warp_sum(w.q != nullptr ? sum_of_piece<T, true>(slot, w.apart, lane) : sum_of_piece<T, false>(slot, 0, lane));
        if (lane == 0) sums[i] = sum;
        __syncwarp();      // (the slot is free)
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// The least token whose inclusive sum of weights exceeds u * (sum of all); -1 if no weight is positive.  By one warp; sum_of(i): a piece's sum.
template <typename T, typename SumOf>
__device__ __forceinline__ int search(const Weights<T>& w, T* slot, SumOf sum_of, int pieces, double u, int lane) {
    // a stretch of pieces to a lane, then the pieces of the stretch
    const int per = (pieces + 31) / 32, c0 = min(lane * per, pieces), c1 = min(c0 + per, pieces);
    double mine = 0.0;
    for (int c = c0; c < c1; ++c) mine += sum_of(c);
    const double upto = warp_scan(mine, lane), total = __shfl_sync(0xffffffffu, upto, 31);
    if (!(total > 0.0)) return -1;
    const double threshold = u * total;
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
    // of the piece: a stretch of its values to a lane (each in an order of its own, so that lanes read different banks), then the values of the stretch
    request_piece(w, slot, piece, lane);
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
    clean_piece(w, slot, piece, lane);
    constexpr int kStretch = kPiece<T> / 32;
    double sum = 0.0;
#pragma unroll 4
    for (int k = 0; k < kStretch; ++k) sum += weight_in(w, slot, lane * kStretch + (k + lane * (4 / (int)sizeof(T))) % kStretch);
    const double end = before + warp_scan(sum, lane);
    const unsigned past = __ballot_sync(0xffffffffu, sum > 0.0 && end > threshold), any = __ballot_sync(0xffffffffu, sum > 0.0);
    const int from = past ? __ffs(past) - 1 : 31 - __clz(any);
    before = __shfl_sync(0xffffffffu, end - sum, from);
    int token = -1;
    for (int k = 0; k < kStretch; k += 32) {
        const double x = weight_in(w, slot, from * kStretch + k + lane), through = before + warp_scan(x, lane);
        const unsigned over = __ballot_sync(0xffffffffu, x > 0.0 && through > threshold), some = __ballot_sync(0xffffffffu, x > 0.0);
        if (some) token = w.token0(piece) + from * kStretch + k + (over ? __ffs(over) - 1 : 31 - __clz(some));
        if (over) break;
        before = __shfl_sync(0xffffffffu, through, 31);
    }
    return token;
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads)
draft_verify_kernel(VerifyArgs a) {
    __shared__ int s_last, s_again;
    extern __shared__ __align__(16) uint8_t s_slots[];
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
                const double pv = probability(bits_of(target[(int64_t)k * a.target_stride + x]));
                const double qv = draft == nullptr ? 1.0 : probability(bits_of(draft[(int64_t)k * a.draft_stride + x]));
                bad = !(probability(bits_of(__ldg(a.accept_u + i0 + k))) * qv < pv);
            }
        }
        const unsigned ballot = __ballot_sync(0xffffffffu, bad);
        if (ballot) {
            accepted = k0 + __ffs(ballot) - 1;
            rejected_token = __shfl_sync(0xffffffffu, x, __ffs(ballot) - 1);
        }
    }
    const bool rejected = accepted < n;
    Weights<T> w(target + (int64_t)accepted * a.target_stride, rejected && draft != nullptr ? draft + (int64_t)accepted * a.draft_stride : nullptr,
                 rejected && draft == nullptr ? rejected_token : -1, a.vocab);
    // ---- this CTA's slice of the row's pieces
    const int slot_values = (a.draft == nullptr ? kSlotBytes : kSlotBytesQ) / (int)sizeof(T);
    T* slots = reinterpret_cast<T*>(s_slots) + (size_t)warp * kSlots * slot_values;
    double* sums = a.sums + (size_t)b * a.pieces;
    const int first = (int)((int64_t)a.pieces * blockIdx.x / gridDim.x), end = (int)((int64_t)a.pieces * (blockIdx.x + 1) / gridDim.x);
    sum_pieces(w, slots, slot_values, first + warp, kVerifyWarps, end, sums, lane);
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
    double* s_sums = reinterpret_cast<double*>(s_slots + (size_t)kSlots * slot_values * sizeof(T));      // the second warp's slots
    int token = -1;
    for (int attempt = 0; attempt < 2; ++attempt) {
        if (shared) {
            for (int i = threadIdx.x; i < a.pieces; i += kVerifyThreads) s_sums[i] = __ldcg(sums + i);
            __syncthreads();
        }
        if (warp == 0) {
            token = search(w, slots, [&](int i) { return shared ? s_sums[i] : __ldcg(sums + i); }, a.pieces, probability(bits_of(__ldg(a.sample_u + b))), lane);
            if (lane == 0) s_again = token < 0 && rejected && attempt == 0;
        }
        __syncthreads();
        if (!s_again) break;
        // nothing is left of max(p - q, 0), as rounded probabilities may have it: the target's own
        w.q = nullptr;
        w.without = -1;
        sum_pieces(w, slots, slot_values, warp, kVerifyWarps, a.pieces, sums, lane);
        __syncthreads();      // (the sums are this CTA's own now)
    }
    if (warp != 0) return;
    for (int k = lane; k <= n; k += 32) a.tokens_out[i0 + b + k] = k < accepted ? __ldg(a.tokens + i0 + k) : k == accepted ? token : -1;
    if (lane == 0) a.accepted[b] = accepted;
}

// CTAs of a kernel that the current device holds at once; asked once for each device and kernel.
cudaError_t ctas_that_fit(void (*kernel)(VerifyArgs), size_t smem, bool wide, bool pairs, int* fit) {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices][4];
    int device = 0, sms = 0, per_sm = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    std::atomic<int>* at = device < kDevices ? &known[device][2 * wide + pairs] : nullptr;
    if (at && (*fit = at->load(std::memory_order_relaxed)) > 0) return cudaSuccess;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kVerifyThreads, smem);
    *fit = sms * per_sm;
    if (e == cudaSuccess && at) at->store(*fit, std::memory_order_relaxed);
    return e;
}

}  // namespace

}  // namespace asynclm

extern "C" size_t asynclm_draft_verify_workspace_bytes(int32_t batch, int32_t vocab) {
    using namespace asynclm;
    if (batch <= 0 || vocab <= 0) return 0;
    const size_t pieces = ((size_t)vocab + 3 + kPiece<float> - 1) / kPiece<float>;      // (rows may start 3 values behind a boundary; of bf16 there are no more)
    return kArrivalBytes + (size_t)batch * pieces * sizeof(double);
}

extern "C" int asynclm_draft_verify(const asynclm_draft_rows* rows, const int32_t* draft_indptr, int32_t batch, int32_t drafts, const int32_t* draft_tokens,
                                    const float* accept_u, const float* sample_u, int32_t* accepted, int32_t* tokens_out, void* workspace, void* stream) {
    using namespace asynclm;
    if (!rows || batch < 0 || drafts < 0 || rows->vocab <= 0 || rows->vocab > INT32_MAX - 4096 || batch > kMostSequences) return ASYNCLM_ERR_INVALID_ARG;
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
    const int piece = size == 4 ? kPiece<float> : kPiece<__nv_bfloat16>;
    a.pieces = (int)(((int64_t)rows->vocab + 16 / (int)size - 1 + piece - 1) / piece);      // wherever a row starts
    const size_t smem = (size_t)kVerifyWarps * kSlots * (rows->draft ? kSlotBytesQ : kSlotBytes);
    auto kernel = size == 4 ? draft_verify_kernel<float> : draft_verify_kernel<__nv_bfloat16>;
    int fit = 0;
    if (int rc = cuda_status(ctas_that_fit(kernel, smem, size == 4, rows->draft != nullptr, &fit))) return rc;
    const int slices = draft_slices(batch, a.pieces, fit, rows->draft != nullptr);
    return cuda_status(launch_pdl(kernel, dim3(slices, batch), dim3(kVerifyThreads), smem, (cudaStream_t)stream, a));
}
