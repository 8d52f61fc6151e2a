// What the kernels of scored steps share: the rows a token sees, and the cap on a score (kvf_scores).
#pragma once
#include <limits.h>
#include <math.h>

#include "kvfold_internal.h"

namespace kvf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct RowRange {
    int64_t begin, end;              // begin >= end: nothing
};
// Rows that token `tok` of a chunk sees of the L rows there are (P of them before the chunk); `at` is its place in the arrays.  Entries
// out of range mean the nearest row there is.
__device__ __forceinline__ RowRange seen_rows(const ScoreMods &m, int64_t at, int tok, int64_t P, int64_t L, int self_rows) {
    RowRange r;
    r.begin = m.first ? (int64_t)max(m.first[at], 0) : 0;
    r.end = m.end ? min((int64_t)max(m.end[at], 0), L) : P + (int64_t)(tok + 1) * self_rows;
    return r;
}

// The cap, softcap * log2(e) * tanh(x) with x = scale / softcap * (q . k).  The special-function unit is what a softmax on the tensor
// cores is short of, so that most scores go through multiply-adds: tanh(x) / x as a polynomial in x^2, of least relative error
// over |x| <= 0.5 (four terms, 5.5e-7) and |x| <= 0.75 (five, 5.7e-7); coefficients by the exchange algorithm of Remez.  Beyond,
// 1 - 2 / (1 + e^2x), whose error of 2^-22 is one of the cap; score by score where one of a warp's tile lies there.
constexpr float kSmallX = 0.5f, kMiddleX = 0.75f;
constexpr double kSmallTanh[4] = {0.9999994557708787, -0.33326317935743466, 0.13190296601601936, -0.044402226090620216};
constexpr double kMiddleTanh[5] = {0.9999994349238549, -0.33328251532272035, 0.13258983219087364, -0.050056302629619055, 0.012929632363192806};
inline void set_cap(ScoreMods &m, double scale, double softcap) {
    const double in = scale / softcap, out = softcap * 1.4426950408889634;
    m.cap_in = (float)in;
    m.cap_out = (float)out;
    m.cap_log2 = (float)(1.0 / out);
    // (powers of `in` outside fp32's range, under caps of a thousand times the usual and far below it: the middle polynomial alone, which
    // does without; tiles of zeros still come by, and zero times these has to be zero)
    const bool powers = in > 1e-4 && in < 1e4;
    m.small_to = powers ? (float)(kSmallX / in) : 0.f;
    for (int i = 0; i < 4; ++i) m.small[i] = powers ? (float)(kSmallTanh[i] * out * pow(in, 2 * i + 1)) : 0.f;
    m.middle_to = (float)(kMiddleX / in);
    for (int i = 0; i < 5; ++i) m.middle[i] = (float)(kMiddleTanh[i] * out);
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 cap_middle(const ScoreMods &m, float2 s) {
    const float2 x = __fmul2_rn(s, both(m.cap_in)), u = __fmul2_rn(x, x);
    float2 y = __ffma2_rn(u, both(m.middle[4]), both(m.middle[3]));
    y = __ffma2_rn(u, y, both(m.middle[2]));
    y = __ffma2_rn(u, y, both(m.middle[1]));
    y = __ffma2_rn(u, y, both(m.middle[0]));
    return __fmul2_rn(x, y);
}
// (s * cap_small_over is the score)
__device__ __forceinline__ float2 cap_small_over(const ScoreMods &m, float2 s) {
    const float2 u = __fmul2_rn(s, s);
    return __ffma2_rn(u, __ffma2_rn(u, __ffma2_rn(u, both(m.small[3]), both(m.small[2])), both(m.small[1])), both(m.small[0]));
}
// x = score / softcap, of a tile where some lie beyond the polynomials
__device__ __forceinline__ float cap_far(const ScoreMods &m, float x) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * (2.f * kLog2e)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return m.cap_out * fmaf(-2.f, r, 1.f);
}
// One score, wherever it lies.  Small ones by the polynomial here too: next to them the error of the other way, 2^-22 of the cap, would
// grow with the cap.
__device__ __forceinline__ float cap_of(const ScoreMods &m, float x) {
    const float u = x * x;
    const float y = x * fmaf(u, fmaf(u, fmaf(u, fmaf(u, m.middle[4], m.middle[3]), m.middle[2]), m.middle[1]), m.middle[0]);
    return fabsf(x) <= kMiddleX ? y : cap_far(m, x);
}
__device__ __forceinline__ float cap_any(const ScoreMods &m, float s) { return cap_of(m, s * m.cap_in); }        // of a dot product
__device__ __forceinline__ float cap_log2(const ScoreMods &m, float y) { return cap_of(m, y * m.cap_log2); }      // of a score in log2 units

}  // namespace
}  // namespace kvf
