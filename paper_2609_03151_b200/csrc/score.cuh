// Shaping of attention scores in registers: the cap c tanh(s / c) and the bias by distance, in log2 units (z log2(e)).
#pragma once
#include "attn_mask.cuh"
#include "ptx.cuh"

namespace {

using namespace ptx;

// tanh(x) = x q(x^2) on |x| <= kTanhNear: interpolation of tanh(sqrt(y)) / sqrt(y) at the five Chebyshev nodes of [0, 1/4] in y,
// relative error below 3e-8 (the next Chebyshev term; the function's nearest pole is at y = -pi^2 / 4).
constexpr float kTanhNear = 0.5f;
constexpr float kTanh1 = -0.33333069f, kTanh2 = 0.13324751f, kTanh3 = -0.052984238f, kTanh4 = 0.017131345f;

__device__ __forceinline__ uint64_t both(float v) { return pack_f2(v, v); }
__device__ __forceinline__ float max3_abs(float a, float b, float c) { return fmaxf(fmaxf(fabsf(a), fabsf(b)), fabsf(c)); }

// q(x^2) of a pair
__device__ __forceinline__ uint64_t tanh_near_q(uint64_t x) {
    const uint64_t y = mul2(x, x);
    uint64_t q = fma2(both(kTanh4), y, both(kTanh3));
    q = fma2(q, y, both(kTanh2));
    q = fma2(q, y, both(kTanh1));
    return fma2(q, y, both(1.f));
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// tanh(x) = 1 - 2 / (exp(2x) + 1): absolute error of a few 2^-24 everywhere, which is what a score of c tanh needs.  The bound keeps
// exp(2x) finite; a NaN passes.
__device__ __forceinline__ float tanh_far(float x) {
    float w = x * 2.8853900817779268f;
    w = w > 64.f ? 64.f : w;
    return fmaf(-2.f, rcp_approx(exp2_approx(w) + 1.f), 1.f);
}

// The 128 scores of a query row against one key tile, raw to log2 units.  dist0: the row's position minus that of the tile's first
// key; side: key tile minus query tile (its sign says on which side of the row all of the keys are).
template <bool kCap, bool kBias>
__device__ __forceinline__ void shape_scores(uint32_t (&s)[128], const ScoreArgs &a, float scale_log2, float slope, int dist0, int side) {
    float sl = 0.f, base = 0.f;
    if constexpr (kBias) {
        sl = side < 0 ? slope : -slope;              // -slope |dist0 - i| = sl i + base on either side of the row
        base = -sl * (float)dist0;
    }
    const uint64_t sl2 = both(sl), base2 = both(base);
    if constexpr (kCap) {
        float top[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 128; i += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) top[k] = max3_abs(top[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
        const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.cap_in;
        if (__any_sync(0xffffffffu, most > kTanhNear)) {
#pragma unroll
            for (int i = 0; i < 128; ++i) {
                float z = tanh_far(__uint_as_float(s[i]) * a.cap_in) * a.cap_out;
                if constexpr (kBias) z += fmaf((float)i, sl, base);
                s[i] = __float_as_uint(z);
            }
        } else {
            const uint64_t in2 = both(a.cap_in), out2 = both(a.cap_out);
#pragma unroll
            for (int i = 0; i < 128; i += 2) {
                const uint64_t x = mul2(pack_f2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), in2);
                const uint64_t q = tanh_near_q(x), w = mul2(x, out2);
                uint64_t z;
                if constexpr (kBias) z = fma2(w, q, fma2(pack_f2((float)i, (float)(i + 1)), sl2, base2));
                else z = mul2(w, q);
                float z0, z1;
                unpack_f2(z, z0, z1);
                s[i] = __float_as_uint(z0);
                s[i + 1] = __float_as_uint(z1);
            }
        }
    } else if constexpr (kBias) {
        const uint64_t sc2 = both(scale_log2);
#pragma unroll
        for (int i = 0; i < 128; i += 2) {
            const uint64_t z = fma2(pack_f2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), sc2,
                                    fma2(pack_f2((float)i, (float)(i + 1)), sl2, base2));
            float z0, z1;
            unpack_f2(z, z0, z1);
            s[i] = __float_as_uint(z0);
            s[i + 1] = __float_as_uint(z1);
        }
    }
    if constexpr (kBias) {
        // the diagonal tile has keys on both sides: those before the row (i < dist0) have the other sign
        if (side == 0) {
#pragma unroll
            for (int i = 0; i < 128; ++i)
                if (i < dist0) s[i] = __float_as_uint(__uint_as_float(s[i]) + 2.f * slope * (float)(i - dist0));
        }
    }
}

}  // namespace
