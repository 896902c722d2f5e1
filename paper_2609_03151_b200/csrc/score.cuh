// Shaping of attention scores in registers: the cap c tanh(s / c) and the bias by distance, in log2 units (z log2(e)).
//
// tanh near zero is an odd polynomial, x (c0 + c1 x^2 + .. + c4 x^8) on |x| <= 0.65: the least largest relative error of that form (1.6e-7, by
// Remez exchange; the function's nearest pole is at x^2 = -pi^2 / 4).  The scale, the cap and
// log2(e) are folded into its coefficients (basp_score_args), so that a raw score s goes to z = s q(s^2).  Elsewhere tanh(x) =
// 1 - 2 / (exp(2x) + 1), whose absolute error of some 2^-24 is what c tanh needs there, at three instead of one operation of the special
// function unit a score.  The fifth coefficient costs 4 % where all scores are near zero (16K causal tokens, 32/8 heads of 128, forward: 1.97 and
// 2.05 ms; up to 0.4 four do) and pays where some are beyond 0.4 (a cap of 10 under scores up to 5.5: 2.18 and 1.81 ms, backward 7.7 and 7.0).
#pragma once
#include <cuda_bf16.h>

#include "attn_mask.cuh"
#include "ptx.cuh"

namespace {

using namespace ptx;

__device__ __forceinline__ uint64_t both(float v) { return pack_f2(v, v); }
__device__ __forceinline__ float round_bf16(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }
__device__ __forceinline__ float max3_abs(float a, float b, float c) { return fmaxf(fmaxf(fabsf(a), fabsf(b)), fabsf(c)); }

// q of a pair of squared raw scores
__device__ __forceinline__ uint64_t cap_near_q(uint64_t y, const ScoreArgs &a) {
    uint64_t q = fma2(both(a.near[4]), y, both(a.near[3]));
    q = fma2(q, y, both(a.near[2]));
    q = fma2(q, y, both(a.near[1]));
    return fma2(q, y, both(a.near[0]));
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// c tanh(s / c) in log2 units for any raw score, to some 2^-23 of the cap, and the cap's derivative 1 - tanh^2 = 4 e r^2 with e = exp(2x),
// r = 1 / (e + 1): no difference of two near numbers where the cap is reached.  The bound keeps e finite; a NaN passes.
__device__ __forceinline__ float capped_far(float s, const ScoreArgs &a, float *derivative) {
    float w = s * a.cap_in * 2.8853900817779268f;
    w = w > 120.f ? 120.f : w;
    const float e = exp2_approx(w), r = rcp_approx(e + 1.f);
    *derivative = 4.f * (e * r) * r;
    return fmaf(-2.f * a.cap_out, r, a.cap_out);
}
// The same to 2^-22 of its own value: a score that is small against the cap by the polynomial
__device__ __forceinline__ float capped_any(float s, const ScoreArgs &a) {
    float derivative;
    const float far = capped_far(s, a, &derivative);
    const float y = s * s, near = s * fmaf(fmaf(fmaf(fmaf(a.near[4], y, a.near[3]), y, a.near[2]), y, a.near[1]), y, a.near[0]);
    return fabsf(s) <= a.near_limit ? near : far;
}

// Raw scores of a query row against neighbouring keys brought to log2 units in place, by the formulas that hold everywhere: where the cap
// is reached, where the bias is steep, where a row has keys on both sides.  dist0: the row's position minus that of the first key.
template <bool kCap, bool kBias, int kCount>
__device__ __forceinline__ void shape_scores(uint32_t (&s)[kCount], const ScoreArgs &a, float scale_log2, float slope, int dist0) {
    const float d0 = (float)dist0;
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
        float z = __uint_as_float(s[i]);
        z = kCap ? capped_any(z, a) : z * scale_log2;
        if constexpr (kBias) z = fmaf(-slope, fabsf(d0 - (float)i), z);
        s[i] = __float_as_uint(z);
    }
}

}  // namespace
