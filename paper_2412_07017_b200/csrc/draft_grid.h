// How the verification of drafted tokens divides its rows among CTAs (draft_verify.cu); host arithmetic only.
#pragma once
#include <algorithm>
#include <cstdint>

namespace asynclm {

constexpr int kVerifyThreads = 64, kVerifyWarps = kVerifyThreads / 32;

// CTAs of a sequence's row of `pieces` pieces; `fit` CTAs fit the GPU at once, 13 to an SM with a draft (by shared memory), 18 without (by registers).
//   As many as half of those that fit, as the next launch's wait beside them: one more and some of its CTAs start late.  Each has a piece or more
// for its warps.  (us out of cache, call after call, with less | so | with more than half: fp32 pairs of 128 256: 64 sequences 17.1 | 16.1 | 18.6,
// 150 27.7 | 25.7 | 30.1, 200 37.3 | 32.9 | 36.5, 237 38.4 | 35.3 | 41.3, 300 51.4 | 44.1 | 49.1; fp32 rows alone: 64 14.5 | 14.0 | 15.1, 128 19.2 | 18.5 | 22.4, 200 25.6 |
// 25.3 | 30.4, 300 35.0 | 35.1 | 42.4; 300 bf16 rows of 100 003 20.8 | 20.3 | 24.7.)
//   One CTA to a row has too little on its way of pairs, so that two are better up to three quarters of those that fit: 356 sequences 83 | 53, 500 86 | 69 (bf16
// 59 | 54), 700 98 | 97 (70 | 63), 888 110 | 117 (72 | 74).  Of rows alone, they are not: 700 77 | 80 (48 | 50), 907 88 | 102 (54 | 60).
inline int draft_slices(int batch, int pieces, int fit, bool pairs) {
    int slices = fit / 2 / batch;
    if (pairs && slices < 2 && (int64_t)2 * batch <= fit * 3 / 4) slices = 2;
    return std::max(1, std::min(slices, (pieces + kVerifyWarps - 1) / kVerifyWarps));
}

}  // namespace asynclm
