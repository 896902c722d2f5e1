// Shaping of attention scores in registers: the cap c tanh(s / c) and the bias by distance, in log2 units (z log2(e)).
//
// tanh near zero is an odd polynomial, x (c0 + c1 x^2 + c2 x^4 + c3 x^6) on |x| <= 0.4: the least largest relative error of that form
// (1e-7, found by iteratively reweighted least squares; the function's nearest pole is at x^2 = -pi^2 / 4).  The scale, the cap and
// log2(e) are folded into its coefficients (basp_score_args), so that a raw score s goes to z = s q(s^2).  Elsewhere tanh(x) =
// 1 - 2 / (exp(2x) + 1), whose absolute error of some 2^-24 is what c tanh needs there.
#pragma once
#include "attn_mask.cuh"
#include "ptx.cuh"

namespace {

using namespace ptx;

__device__ __forceinline__ uint64_t both(float v) { return pack_f2(v, v); }
__device__ __forceinline__ float max3_abs(float a, float b, float c) { return fmaxf(fmaxf(fabsf(a), fabsf(b)), fabsf(c)); }

// q of a pair of squared raw scores
__device__ __forceinline__ uint64_t cap_near_q(uint64_t y, const ScoreArgs &a) {
    uint64_t q = fma2(both(a.near[3]), y, both(a.near[2]));
    q = fma2(q, y, both(a.near[1]));
    return fma2(q, y, both(a.near[0]));
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// tanh of any x.  The bound keeps exp(2x) finite; a NaN passes.
__device__ __forceinline__ float tanh_far(float x) {
    float w = x * 2.8853900817779268f;
    w = w > 64.f ? 64.f : w;
    return fmaf(-2.f, rcp_approx(exp2_approx(w) + 1.f), 1.f);
}

// Raw scores of a query row against neighbouring keys brought to log2 units in place, by the formulas that hold everywhere: where the cap
// is reached, where the bias is steep, where a row has keys on both sides.  dist0: the row's position minus that of the first key.
template <bool kCap, bool kBias, int kCount>
__device__ __forceinline__ void shape_scores(uint32_t (&s)[kCount], const ScoreArgs &a, float scale_log2, float slope, int dist0) {
    const float d0 = (float)dist0;
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
        float z = __uint_as_float(s[i]);
        z = kCap ? tanh_far(z * a.cap_in) * a.cap_out : z * scale_log2;
        if constexpr (kBias) z = fmaf(-slope, fabsf(d0 - (float)i), z);
        s[i] = __float_as_uint(z);
    }
}

}  // namespace
