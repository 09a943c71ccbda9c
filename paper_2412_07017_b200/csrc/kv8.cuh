// The 8-bit cache's number format on the device (host side and layout: include/asynclm.h, "Quantised cache").
//
// A row (head_dim values of one token, kv head and K or V) is held as e4m3 codes and one power of two:
//     x_j ~ c_j * 2^e,   c_j = e4m3 nearest to x_j * 2^-e,   e = the least integer >= -100 with max|x_j| <= 448 * 2^e.
// Why a power of two: e4m3 is a floating-point format, whose relative step is 2^-4 wherever a value lies, so a scale
// that brings the maximum to 448 exactly gains nothing but up to one more bit at the subnormal end (values below 2^-6 *
// 2^e).  For it, x * 2^-e and c * 2^e are exact (the only rounding is that of the code) and c * 2^e is a bf16 value, so
// reading back rounds nothing; scores are taken on the codes, whose 2^e of K multiplies the finished product; V is
// taken times 2^(e - a reference's), which shifts exponents alone; and a scale is one byte (e8m0: e + 127), 1/128 of
// its row at head_dim 128.
// Why e >= -100: c * 2^e then stays clear of fp32's and bf16's subnormal numbers, which these kernels flush; values
// below 2^-110 become zeros.
#pragma once
#include <cuda_fp16.h>
#include <stdint.h>

#include "common.cuh"

namespace asynclm {

constexpr int kKv8LeastExponent = -100;
constexpr uint32_t kKv8NanByte = 255;      // scale of a row with a value that is not finite; its codes are zeros
constexpr int kKv8ScaleBytes = 2 * kPage;  // of one (page, kv head): 16 K rows, 16 V rows
constexpr int kStatusBadGather = 45;
// The attention kernels hold a key's weight, exp2(score + eV - reference), as an f16 number, times 2^kKv8WeightShift:
// the reference may be exceeded by 2^8, so they stay below 2^15, and one loses bits only where it is below 2^-21 of the
// reference's weight and counts as zero below 2^-32.
constexpr int kKv8WeightShift = 7;

// Byte offset of the codes of (page, K|V, kv head, slot), and of its scale byte.
__device__ __forceinline__ size_t kv8_row_offset(int64_t page, int which, int kv_head, int slot, int num_kv_heads, int head_dim) {
    return pool_row_offset(page, which, kv_head, slot, num_kv_heads, head_dim);      // (one byte a value)
}
__device__ __forceinline__ size_t kv8_scale_offset(int64_t page, int which, int kv_head, int slot, int num_kv_heads) {
    return ((size_t)page * (size_t)num_kv_heads + (size_t)kv_head) * kKv8ScaleBytes + (size_t)(which * kPage + slot);
}

// 2^(byte - 127); the byte 255 is NaN, the byte 0 (which no append writes) counts as zero.
__device__ __forceinline__ float kv8_scale(uint32_t byte) {
    return __uint_as_float(byte == kKv8NanByte ? 0x7fffffffu : byte << 23);
}

// Biased exponent byte of the row whose largest magnitude has the fp32 bits `most` (sign cleared; NaN and infinity are
// the largest): 448 is 1.75 * 2^8.
__device__ __forceinline__ uint32_t kv8_scale_byte(uint32_t most) {
    if (most >= 0x7f800000u) return kKv8NanByte;
    const int e = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, kKv8LeastExponent + 127);
}

// Two values -> two codes (lo in the low byte).  The values are within +-448 here; cvt's saturation has nothing to do.
__device__ __forceinline__ uint32_t kv8_encode2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// Two codes (the low byte first) -> two f16 values, exact.
__device__ __forceinline__ uint32_t kv8_decode2(uint32_t codes) {
    uint32_t r;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(r) : "r"(codes));
    return r;
}
__device__ __forceinline__ uint32_t kv8_decode2_hi(uint32_t codes) {      // of the upper half
    uint32_t r;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, b;\n\t}" : "=r"(r) : "r"(codes));
    return r;
}

}  // namespace asynclm
