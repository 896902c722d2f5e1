// Rotary positions of Q and K on all ranks' sequence shards, with a position of its own for every token (packed documents restart it),
// in half or interleaved pairs, over part of the head, with frequencies scaled for long contexts.
//
//   (x_u, x_v) -> factor (x_u cos a - x_v sin a,  x_v cos a + x_u sin a),  a = position theta_j
//
// The frequencies are 64-bit fixed-point turns per token: position x frequency in 64-bit integers drops whole turns by itself, and
// the fraction that is left is good to 2^-32 of a turn at any position (2^-26, some 10^-7 radian, once it is the fp32 argument of the sine
// and cosine), where fp32 throughout (2^-24 of the angle) is 0.01 radian off at 128K.  So a lane makes
// its eight angles from the position alone (an integer product and a sine and a cosine each) and no table is read.
//
// HBM-bound: 2 bytes read and 2 written per element.  A lane holds two vectors of 16 bytes, D / 16 lanes a head: in the half layout the two
// halves of eight pairs or two vectors that are only copied, interleaved one of each half of the head.  Neighbouring lanes have
// neighbouring vectors, so every access is of whole sectors (a lane with sixteen neighbouring features reads each twice: 64K tokens
// interleaved 234 us, against 205).  A warp holds 32 / (D / 16) heads of one token, Q's and K's in one list, so the angles are made once for a
// token's share of heads.  80 registers, three blocks per SM: 64K tokens, 40 heads of 128: 206 us (6.5 TB/s); at 96 registers and two blocks 228 us.
#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"
#include "spans.h"

namespace {

using namespace ptx;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 4;             // heads in flight per lane: 128 bytes

// R: room for ranks (8 or BASP_MAX_RANKS; a launch takes longer the larger its parameters)
template <int R>
struct RopeParams {
    const __nv_bfloat16 *q[R], *k[R];
    __nv_bfloat16 *q_out[R], *k_out[R];
    const int *positions;      // [B][S], or nullptr
    unsigned long long turns[64];
    float factor, sign;        // sign: -1 for the inverse
    int D, S, T, T_last, K, Bl, Hq, H;            // H: heads of Q and K
    int half, rotary, interleaved;
    uint32_t chunks, chunk_heads;                 // a token's heads in chunks (a warp's work)
    uint32_t rows, items;                         // rows: of a full rank; items: warps' worth of work
    FastDiv div_chunks, div_rows, div_T, div_T_last, div_K;
};

__device__ __forceinline__ uint4 ld16(const __nv_bfloat16 *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void st16(__nv_bfloat16 *p, const uint4 &v) {
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" :: "l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Eight pairs whose halves are in two vectors
__device__ __forceinline__ void turn_halves(uint4 &a, uint4 &b, const float (&c)[8], const float (&s)[8]) {
    uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float u0 = low(x[i]), u1 = high(x[i]), v0 = low(y[i]), v1 = high(y[i]);
        const int e = 2 * i;
        x[i] = pack_bf16x2(fmaf(u0, c[e], -(v0 * s[e])), fmaf(u1, c[e + 1], -(v1 * s[e + 1])));
        y[i] = pack_bf16x2(fmaf(v0, c[e], u0 * s[e]), fmaf(v1, c[e + 1], u1 * s[e + 1]));
    }
    a = make_uint4(x[0], x[1], x[2], x[3]);
    b = make_uint4(y[0], y[1], y[2], y[3]);
}
// Four pairs side by side; their angles start at `first`
template <int first>
__device__ __forceinline__ void turn_pairs(uint4 &a, const float (&c)[8], const float (&s)[8]) {
    uint32_t x[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float u = low(x[i]), v = high(x[i]);
        x[i] = pack_bf16x2(fmaf(u, c[first + i], -(v * s[first + i])), fmaf(v, c[first + i], u * s[first + i]));
    }
    a = make_uint4(x[0], x[1], x[2], x[3]);
}

// N = D / 16 lanes hold a head
template <int N, int R>
__global__ void __launch_bounds__(kThreads, 3) rope_kernel(const __grid_constant__ RopeParams<R> p) {
    constexpr int kHeads = 32 / N;     // heads of a warp's step
    const int warp_lane = threadIdx.x & 31, slot = warp_lane / N, lane = warp_lane - slot * N;
    const uint32_t item = blockIdx.x * kWarps + threadIdx.x / 32;
    if (item >= p.items || slot >= kHeads) return;
    const uint32_t token = fdiv(item, p.div_chunks), chunk = item - token * p.chunks;      // token: of all ranks, full ones
    const uint32_t r = fdiv(token, p.div_rows), row = token - r * p.rows;
    const uint32_t g = fdiv(r, p.div_K), l = r - g * p.K;
    const bool last = (int)l == p.K - 1;
    const uint32_t Tr = last ? p.T_last : p.T;
    if (row >= p.Bl * Tr) return;      // a short last rank
    const uint32_t bl = fdiv(row, last ? p.div_T_last : p.div_T), place = l * p.T + (row - bl * Tr);
    // the lane's two vectors, and which of them are rotated
    const int turned = p.rotary / 16;                          // half layout: lanes with pairs
    int at = 8 * lane, other = at + 8 * N;
    bool turn_a = at < p.rotary, turn_b = other < p.rotary;    // interleaved
    if (!p.interleaved) {
        turn_a = turn_b = lane < turned;
        if (!turn_a) at = p.rotary + 8 * (lane - turned);
        other = at + (turn_a ? p.half : 8 * (N - turned));
    }
    const int first = (int)(chunk * p.chunk_heads), past = min(first + (int)p.chunk_heads, p.H);
    const __nv_bfloat16 *q = p.q[r] + (size_t)row * p.Hq * p.D, *k = p.k[r] + (size_t)row * (p.H - p.Hq) * p.D;
    __nv_bfloat16 *qo = p.q_out[r] + (size_t)row * p.Hq * p.D, *ko = p.k_out[r] + (size_t)row * (p.H - p.Hq) * p.D;
    float c[8], s[8];
    for (int h0 = first + slot; h0 < past; h0 += kUnroll * kHeads) {
        uint4 a[kUnroll], b[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = h0 + u * kHeads;
            if (h < past) {
                const __nv_bfloat16 *x = h < p.Hq ? q + (size_t)h * p.D : k + (size_t)(h - p.Hq) * p.D;
                a[u] = ld16(x + at);
                b[u] = ld16(x + other);
            }
        }
        if (h0 == first + slot && (turn_a || turn_b)) {        // behind the first loads: their latencies overlap
            const long long pos = p.positions ? (long long)__ldg(p.positions + (size_t)(g * p.Bl + bl) * p.S + place) : (long long)place;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // the fraction of a turn as a signed 32-bit number, halves of a turn as sincospi takes them
                const int pair = p.interleaved ? (e < 4 ? 4 * lane + e : 4 * (lane + N) + e - 4) : 8 * lane + e;      // (below D / 2)
                const unsigned long long t = (unsigned long long)pos * p.turns[pair];
                float sn, cs;
                sincospif((float)(int)(t >> 32) * 4.656612873077393e-10f, &sn, &cs);
                c[e] = cs * p.factor;
                s[e] = sn * p.factor * p.sign;
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = h0 + u * kHeads;
            if (h < past) {
                if (!p.interleaved) {
                    if (turn_a) turn_halves(a[u], b[u], c, s);
                } else {
                    if (turn_a) turn_pairs<0>(a[u], c, s);
                    if (turn_b) turn_pairs<4>(b[u], c, s);
                }
                __nv_bfloat16 *y = h < p.Hq ? qo + (size_t)h * p.D : ko + (size_t)(h - p.Hq) * p.D;
                st16(y + at, a[u]);
                st16(y + other, b[u]);
            }
        }
    }
}

// f(the number as a type) for one of the listed numbers
template <int... kN, typename F>
int dispatch(int n, F &&f) {
    int rc = BASP_ERR_UNSUPPORTED;
    ((n == kN ? (void)(rc = f(std::integral_constant<int, kN>{})) : (void)0), ...);
    return rc;
}

template <int R>
int run(const basp_plan *pl, const basp_rope_turns *rope, const void *const *q_seq, const void *const *k_seq, const int *positions,
        int inverse, void *const *q_out, void *const *k_out, void *stream) {
    RopeParams<R> prm;
    SpanSet spans;
    for (int r = 0; r < pl->N; ++r) {
        const size_t rows = (size_t)pl->Bl * basp_rank_tokens(pl, r % pl->K), qb = rows * pl->Hq * pl->D * 2, kb = rows * pl->Hkv * pl->D * 2;
        BASP_TRY(spans.add_in(q_seq[r], qb, 16, r));
        BASP_TRY(spans.add_in(k_seq[r], kb, 16, BASP_MAX_RANKS + r));
        BASP_TRY(spans.add_out(q_out[r], qb, 16, r));
        BASP_TRY(spans.add_out(k_out[r], kb, 16, BASP_MAX_RANKS + r));
        prm.q[r] = (const __nv_bfloat16 *)q_seq[r]; prm.k[r] = (const __nv_bfloat16 *)k_seq[r];
        prm.q_out[r] = (__nv_bfloat16 *)q_out[r]; prm.k_out[r] = (__nv_bfloat16 *)k_out[r];
    }
    if (positions) BASP_TRY(spans.add_in(positions, (size_t)pl->B * pl->S * 4, 4));
    BASP_TRY(spans.overlaps());
    prm.positions = positions;
    for (int j = 0; j < 64; ++j) prm.turns[j] = rope->turns[j];
    prm.factor = rope->factor; prm.sign = inverse ? -1.f : 1.f;
    prm.D = pl->D; prm.S = pl->S; prm.T = pl->T; prm.T_last = pl->T_last; prm.K = pl->K; prm.Bl = pl->Bl;
    prm.Hq = pl->Hq; prm.H = pl->Hq + pl->Hkv;
    prm.half = rope->rotary_dim / 2; prm.rotary = rope->rotary_dim; prm.interleaved = rope->interleaved;
    const int lanes = pl->D / 16, step = kUnroll * (32 / lanes);          // heads of a warp's step
    const long long rows = (long long)pl->Bl * pl->T, tokens = rows * pl->N;
    // A token's heads as one warp's work, so that its angles are made once; where the tokens do not fill the GPU (148 SMs of some 48
    // warps) one step of heads a warp
    const long long steps = (prm.H + step - 1) / step;
    prm.chunk_heads = tokens >= 148 * 48 ? (uint32_t)(steps * step) : (uint32_t)step;
    prm.chunks = (uint32_t)((prm.H + prm.chunk_heads - 1) / prm.chunk_heads);
    const long long items = tokens * prm.chunks;
    if (items >= (1ll << 31) - kWarps) return BASP_ERR_UNSUPPORTED;
    prm.rows = (uint32_t)rows; prm.items = (uint32_t)items;
    prm.div_chunks = make_fastdiv(prm.chunks); prm.div_rows = make_fastdiv(prm.rows); prm.div_K = make_fastdiv((uint32_t)pl->K);
    prm.div_T = make_fastdiv((uint32_t)pl->T); prm.div_T_last = make_fastdiv((uint32_t)pl->T_last);
    return dispatch<1, 2, 3, 4, 5, 6, 7, 8>(lanes, [&](auto n) -> int {
        rope_kernel<decltype(n)::value, R><<<(unsigned)((items + kWarps - 1) / kWarps), kThreads, 0, (cudaStream_t)stream>>>(prm);
        BASP_CUDA_TRY(cudaGetLastError());
        basp_count_launch(1);
        return BASP_OK;
    });
}

bool rotary_ok(int n) { return n >= 16 && n <= 128 && n % 16 == 0; }

}  // namespace

extern "C" int basp_rope_make(const basp_rope_config *c, basp_rope_turns *out) {
    if (!c || !out) return BASP_ERR_NULL;
    if (!rotary_ok(c->rotary_dim)) return BASP_ERR_UNSUPPORTED;
    if (c->scaling < BASP_ROPE_PLAIN || c->scaling > BASP_ROPE_WAVELENGTH) return BASP_ERR_INVALID;
    if (!(c->base > 1.0 && c->base <= 1e30)) return BASP_ERR_INVALID;
    if (!(c->factor >= 0.0 && c->factor <= 1e30)) return BASP_ERR_INVALID;
    // in 80 bits where the host has them: at position 2^31 the 53 bits of a double would leave 2^-25 of a turn
    typedef long double wide;
    const wide two_pi = 6.283185307179586476925286766559L;
    const bool parts = c->scaling == BASP_ROPE_BY_PARTS, waves = c->scaling == BASP_ROPE_WAVELENGTH;
    double slow = c->slow, fast = c->fast;
    if (c->scaling != BASP_ROPE_PLAIN && !(c->stretch >= 1.0 && c->stretch <= 1e30)) return BASP_ERR_INVALID;
    if (parts || waves) {
        if (!(c->original_len >= 1.0 && c->original_len <= 1e30)) return BASP_ERR_INVALID;
        if (slow == 0.0 && fast == 0.0) { slow = 1.0; fast = parts ? 32.0 : 4.0; }
        if (!(slow > 0.0 && fast > slow && fast <= 1e30)) return BASP_ERR_INVALID;
    }
    *out = basp_rope_turns{};
    out->rotary_dim = c->rotary_dim;
    out->interleaved = c->interleaved != 0;
    double factor = c->factor;
    if (factor == 0.0) factor = parts ? 0.1 * log(c->stretch) + 1.0 : 1.0;
    out->factor = (float)factor;
    const int half = c->rotary_dim / 2;
    // BY_PARTS: the pair numbers whose frequencies turn `fast` and `slow` times in the trained length, rounded outwards
    double first = 0.0, last = 0.0;
    if (parts) {
        first = floor(half * log(c->original_len / (fast * (double)two_pi)) / log(c->base));
        last = ceil(half * log(c->original_len / (slow * (double)two_pi)) / log(c->base));
        if (first < 0.0) first = 0.0;
        if (last > c->rotary_dim - 1.0) last = c->rotary_dim - 1.0;
        if (last - first < 0.001) last = first + 0.001;
    }
    for (int j = 0; j < half; ++j) {
        wide per_token = powl((wide)c->base, -(wide)j / half) / two_pi;     // in turns
        wide keep = 1.0L;                                                   // share of the trained frequency
        if (c->scaling == BASP_ROPE_LINEAR) keep = 0.0L;
        if (parts) keep = 1.0L - (j - (wide)first) / ((wide)last - first);
        if (waves) keep = (c->original_len * per_token - slow) / ((wide)fast - slow);
        keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
        if (c->scaling != BASP_ROPE_PLAIN) per_token = per_token * keep + per_token / c->stretch * (1.0L - keep);
        out->turns[j] = (unsigned long long)(ldexpl(per_token, 64) + 0.5L);           // below 1 / 2 pi: fits
    }
    return BASP_OK;
}

extern "C" int basp_rope(const basp_plan *p, const basp_rope_turns *rope, const void *const *q_seq, const void *const *k_seq,
                         const int *positions, int inverse, void *const *q_out, void *const *k_out, void *stream) {
    if (!p || !rope || !q_seq || !k_seq || !q_out || !k_out) return BASP_ERR_NULL;
    if (p->D % 16 != 0 || p->D > 128) return BASP_ERR_UNSUPPORTED;
    if (!rotary_ok(rope->rotary_dim) || rope->rotary_dim > p->D) return BASP_ERR_UNSUPPORTED;
    if (!(rope->factor > 0.f && rope->factor <= 1e30f)) return BASP_ERR_INVALID;
    return p->N <= 8 ? run<8>(p, rope, q_seq, k_seq, positions, inverse, q_out, k_out, stream)
                     : run<BASP_MAX_RANKS>(p, rope, q_seq, k_seq, positions, inverse, q_out, k_out, stream);
}
