// Backward of the attention with masked and shaped scores (attn_masked_fwd.cu) over each virtual rank's head slice:
//
//   P_ij = exp(z_ij - LSE_i) on visible pairs,  Delta_i = dO_i.O_i (= sum_j P_ij dO_i.v_j),  dV_j = sum_i P_ij dO_i,
//   dZ_ij = P_ij (dO_i.v_j - Delta_i),  dS_ij = scale (1 - tanh^2(scale q_i.k_j / c)) dZ_ij,  dQ_i = sum_j dS_ij k_j,  dK_j = sum_i dS_ij q_i
//
// The kernels are those of attn_bwd.cu (five products per tile pair on tcgen05, dK and dV resident in TMEM, dQ added to an fp32
// accumulator), walking the tile pairs of the mask object: a work item is a key tile and the query tiles that see some of it,
// longest first.  A row without a key has LSE = -inf and takes no part; a key tile that nothing sees gets zeros.
// P and dS become bf16 as operands of the products (the tensor cores take no wider ones at their full rate), everything else is fp32 up to the
// results: dQ and dK are off by 0.0025 to 0.0029 (2-norm; 0.0017 for the exact result rounded), by up to 0.005 in a shard where few keys of
// more than eight have a query's weight (short windows, steep slopes, large scores) and the roundings of P and O in Delta count (mb_prepare_kernel).
// 16K causal tokens, 32/8 heads of 128: plain 5.4-5.6 ms (1000 TFLOP/s, as the causal kernel), through a mask object 5.96-6.1 (the tile's entry and
// the rows' ranges, loaded and staged at every step), bias 5.7-5.9, cap 50 6.9-7.0, both 6.9-7.0.  The tensor pipe is busy for half of the time
// on packed documents; the rest is instruction fetch, the chain of a step's products and the reductions of dQ.
#include <cuda.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"
#include "tmap.cuh"
#include "attn_bwd_common.cuh"
#include "attn_mask.cuh"
#include "score.cuh"
#include "spans.h"

int *basp_status_device_ptr();

namespace {

template <int R>
struct MaskedBwdParams {
    CUtensorMap q[R], k[R], v[R], dout[R];
    CUtensorMap dq_acc[R];      // fp32 accumulator, box 32 floats x 1 head x 32 rows (reduce-add target of the 64-wide kernel)
    float *dq_accp[R];          // the same accumulator as a plain pointer ([Bl*S][Hq_l][Dg] floats)
    const float *lse[R];
    const float *delta[R];
    __nv_bfloat16 *dk[R], *dv[R];
    __nv_bfloat16 *dq[R];       // written at once where a sequence is one key tile (direct)
    float *kv_part;             // [rank][part][dK, dV][kv_elems]: where the query heads of a key head are divided
    size_t kv_elems;
    int parts, part_heads, direct;
    ScoreArgs score;
    int K, Bl, S, Hq_l, Hkv_l, q_per_kv, causal, n_tiles, total;      // total: work items
    int Dg;                     // head dimension in memory
    float scale, scale_log2;
    int *status;
    FastDiv div_items, div_parts, div_hkv_l, div_B, div_bl;
};

struct MbItem {
    int r, bl, seq, hkv, n, m0, n_qt;
    int part;                   // which part of the key head's query heads (see mb_heads)
};

// kSmall: the query heads of a key head may be divided (parts), and dQ may leave at once (direct).  A variant of its own: in one, the
// code for both cost the large plans a tenth (16K causal tokens: 5.6 and 6.2 ms).
template <bool kSmall, int R>
__device__ __forceinline__ bool mb_get_item(const MaskedBwdParams<R> &p, int round, MbItem &it) {
    const int pos = (round & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x;   // boustrophedon
    const int i = round * (int)gridDim.x + pos;
    if (i >= p.total) return false;
    const int e = (int)fdiv((uint32_t)i, p.div_items), head = i - e * (int)p.div_items.d;
    const int lh = kSmall ? (int)fdiv((uint32_t)head, p.div_parts) : head, l = (int)fdiv((uint32_t)lh, p.div_hkv_l);
    it.part = kSmall ? head - lh * p.parts : 0;
    it.hkv = lh - l * p.Hkv_l;
    if (p.score.range) {
        const int4 a = __ldg(reinterpret_cast<const int4 *>(p.score.bwd + e));
        it.seq = min(max(a.x, 0), p.score.B - 1);       // whatever the buffer holds, no tile outside the tensors
        it.n = min(max(a.y, 0), p.n_tiles - 1);
        it.m0 = max(a.z, 0);
        it.n_qt = min(a.w, p.n_tiles);
    } else {
        it.n = (int)fdiv((uint32_t)e, p.div_B);          // low key tiles are seen by the most query tiles: longest first
        it.seq = e - it.n * p.score.B;
        it.m0 = p.causal ? it.n : 0;
        it.n_qt = p.n_tiles;
    }
    const int g = (int)fdiv((uint32_t)it.seq, p.div_bl);
    it.bl = it.seq - g * p.Bl;
    it.r = g * p.K + l;
    return true;
}

// Query heads of an item, and the first of them among the rank's
template <bool kSmall, int R>
__device__ __forceinline__ int mb_heads(const MaskedBwdParams<R> &p, const MbItem &it) {
    return kSmall ? min(p.part_heads, p.q_per_kv - it.part * p.part_heads) : p.q_per_kv;
}
template <bool kSmall, int R>
__device__ __forceinline__ int mb_first_head(const MaskedBwdParams<R> &p, const MbItem &it) {
    return it.hkv * p.q_per_kv + (kSmall ? it.part * p.part_heads : 0);
}

// A query's LSE in log2 units; one that sees no key gets the LSE at which every probability is zero.
__device__ __forceinline__ float seen_lse(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

// What the producer warp brings for a query tile besides Q and dO, four queries a lane: LSE and Delta, and which rows [lo, hi) of the key
// tile they see.
struct MbStats {
    float4 lse, delta;
    int4 tile, range[2];
};
template <int R>
__device__ __forceinline__ MbStats fetch_stats(const MaskedBwdParams<R> &p, const MbItem &it, int h, int m, int lane) {
    MbStats s;
    const size_t off = ((size_t)it.bl * p.Hq_l + h) * p.S + (size_t)m * kT + 4 * lane;
    if ((p.S & 3) == 0 && (m + 1) * kT <= p.S) {
        s.lse = *reinterpret_cast<const float4 *>(p.lse[it.r] + off);
        s.delta = *reinterpret_cast<const float4 *>(p.delta[it.r] + off);
    } else {                       // ragged: rows of (bl, h) are not 16-byte aligned, or the tile runs past S
        float lv[4], dv[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool in_seq = m * kT + 4 * lane + e < p.S;
            lv[e] = in_seq ? p.lse[it.r][off + e] : 0.f;
            dv[e] = in_seq ? p.delta[it.r][off + e] : 0.f;
        }
        s.lse = make_float4(lv[0], lv[1], lv[2], lv[3]);
        s.delta = make_float4(dv[0], dv[1], dv[2], dv[3]);
    }
    if (p.score.range) {
        const size_t tile = (size_t)it.seq * p.n_tiles + m;
        s.tile = __ldg(reinterpret_cast<const int4 *>(p.score.tiles + tile));
        const int4 *at = reinterpret_cast<const int4 *>(p.score.range + tile * kT + 4 * lane);
        s.range[0] = __ldg(at);
        s.range[1] = __ldg(at + 1);
    }
    return s;
}
// To shared memory: LSE in log2 units, -Delta times the scale, the windows, and whether the windows are to be looked at (bit 0 of edge).  A
// window is lo | hi << 8 in keys of the tile, both 0 where there are none, with bit 7 where the query sees one key in all (bit 1 + g of edge:
// one of queries 32 g .. + 31 does).
template <int R>
__device__ __forceinline__ void stage_stats(const MaskedBwdParams<R> &p, const MbItem &it, int m, int lane, const MbStats &s, float *lse,
                                            float *delta, uint16_t *win, int *edge) {
    *reinterpret_cast<float4 *>(lse + 4 * lane) = make_float4(seen_lse(s.lse.x), seen_lse(s.lse.y), seen_lse(s.lse.z), seen_lse(s.lse.w));
    *reinterpret_cast<float4 *>(delta + 4 * lane) = make_float4(s.delta.x * -p.scale, s.delta.y * -p.scale, s.delta.z * -p.scale, s.delta.w * -p.scale);
    const int k0 = it.n * kT;
    int lo[4], hi[4];
    bool look;
    if (p.score.range) {
        look = it.n < s.tile.z || it.n >= s.tile.w || (m + 1) * kT > p.S;
        lo[0] = s.range[0].x; hi[0] = s.range[0].y; lo[1] = s.range[0].z; hi[1] = s.range[0].w;
        lo[2] = s.range[1].x; hi[2] = s.range[1].y; lo[3] = s.range[1].z; hi[3] = s.range[1].w;
    } else {
        look = (p.causal && m == it.n) || (m + 1) * kT > p.S || (it.n + 1) * kT > p.S;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int q = m * kT + 4 * lane + e;
            lo[e] = 0;
            hi[e] = q < p.S ? (p.causal ? q + 1 : p.S) : 0;
        }
    }
    uint32_t w[4];
    bool single = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int first = max(lo[e] - k0, 0), past = min(hi[e] - k0, kT);
        const bool one = first < past && hi[e] - lo[e] == 1;
        w[e] = first < past ? (uint32_t)(first | past << 8 | (one ? 0x80 : 0)) : 0u;
        single = single || one;
    }
    *reinterpret_cast<uint2 *>(win + 4 * lane) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    const uint32_t singles = __ballot_sync(0xffffffffu, single);
    if (lane == 0)
        *edge = look | (singles & 0xff ? 2 : 0) | (singles & 0xff00 ? 4 : 0) | (singles & 0xff0000 ? 8 : 0) | (singles & 0xff000000u ? 16 : 0);
}

// Thirty-two scores of a key row (queries side by side): the probabilities as bf16 to the tensor memory at `to`, sixteen at a time, and
// times the cap's derivative to st.
// dist: the first query's position minus the key's; side: its sign, tile by tile; win: what stage_stats left, where it matters.
template <bool kCap, bool kBias, bool kEdge>
__device__ __forceinline__ void shaped_probs(uint32_t (&st)[32], uint32_t to, const float *lse, const uint16_t *win, int row,
                                             const ScoreArgs &a, float scale_log2, float slope, int dist, int side) {
    [[maybe_unused]] float sl = 0.f, base = 0.f;
    if constexpr (kBias) {
        sl = side < 0 ? slope : -slope;              // -slope |dist + c| = sl c + base on either side of the key
        base = sl * (float)dist;
    }
    [[maybe_unused]] const uint64_t shrink = both(-1.f / (a.cap_out * a.cap_out));
    const uint64_t minus2 = both(-1.f);
    [[maybe_unused]] bool far = false;
    if constexpr (kCap) {
        float top[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 32; c += 4)
#pragma unroll
            for (int k = 0; k < 2; ++k) top[k] = max3_abs(top[k], __uint_as_float(st[c + 2 * k]), __uint_as_float(st[c + 2 * k + 1]));
        far = __any_sync(0xffffffffu, fmaxf(top[0], top[1]) > a.near_limit);
    }
    [[maybe_unused]] uint64_t ramp[2], block = 0;    // the bias of pair c as ramp + block: no constants in the code
    if constexpr (kBias) {
        ramp[0] = pack_f2(0.f, sl);
        ramp[1] = pack_f2(2.f * sl, 3.f * sl);
    }
    const auto columns = [&](auto far_tag) {
        [[maybe_unused]] constexpr bool kFar = decltype(far_tag)::value;
        uint32_t pk[8];
#pragma unroll
        for (int c = 0; c < 32; c += 4) {
            const float4 l4 = *reinterpret_cast<const float4 *>(lse + c);
            uint2 w4 = make_uint2(0, 0);
            if constexpr (kEdge) w4 = *reinterpret_cast<const uint2 *>(win + c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = c + 2 * h;
                uint64_t off = h ? pack_f2(l4.z, l4.w) : pack_f2(l4.x, l4.y);          // -LSE and the bias
                if constexpr (kBias) {
                    if (h == 0) block = both(fmaf(sl, (float)c, base));
                    off = fma2(off, minus2, add2(ramp[h], block));
                } else off = mul2(off, minus2);
                const uint64_t s2 = pack_f2(__uint_as_float(st[i]), __uint_as_float(st[i + 1]));
                [[maybe_unused]] uint64_t slope2 = 0;          // the cap's derivative
                uint64_t z;
                if constexpr (!kCap) {
                    z = fma2(s2, both(scale_log2), off);
                } else if constexpr (kFar) {
                    float g0, g1;
                    const float c0 = capped_far(__uint_as_float(st[i]), a, &g0), c1 = capped_far(__uint_as_float(st[i + 1]), a, &g1);
                    z = add2(pack_f2(c0, c1), off);
                    slope2 = pack_f2(g0, g1);
                } else {
                    const uint64_t q = cap_near_q(mul2(s2, s2), a), capped = mul2(s2, q);
                    z = fma2(s2, q, off);
                    slope2 = fma2(mul2(capped, capped), shrink, both(1.f));
                }
                float z0, z1;
                unpack_f2(z, z0, z1);
                if constexpr (kBias && kEdge) {       // the diagonal tile has queries on both sides of the key
                    if (side == 0) {
                        z0 = fmaf(2.f * slope, fminf((float)dist + (float)i, 0.f), z0);
                        z1 = fmaf(2.f * slope, fminf((float)dist + (float)(i + 1), 0.f), z1);
                    }
                }
                float p0 = exp2_approx(z0), p1 = exp2_approx(z1);
                if constexpr (kEdge) {
                    const uint32_t w = h ? w4.y : w4.x;
                    if (!(row >= (int)(w & 0x7f) && row < (int)((w >> 8) & 0xff))) p0 = 0.f;
                    if (!(row >= (int)((w >> 16) & 0x7f) && row < (int)(w >> 24))) p1 = 0.f;
                }
                pk[(i >> 1) & 7] = pack_bf16x2(p0, p1);
                if constexpr (kBias && kEdge) {       // drop_singles, without a loop of its own
                    const uint32_t w = h ? w4.y : w4.x;
                    if (w & 0x80) p0 = 0.f;
                    if (w & 0x800000) p1 = 0.f;
                }
                if constexpr (kCap) unpack_f2(mul2(pack_f2(p0, p1), slope2), p0, p1);
                st[i] = __float_as_uint(p0);
                st[i + 1] = __float_as_uint(p1);
            }
            if (c % 16 == 12) tmem_st_x8(to + c / 16 * 8, pk);
        }
    };
    if constexpr (kCap) {
        if (far) columns(std::true_type{});
        else columns(std::false_type{});
    } else {
        columns(std::false_type{});
    }
}

// A query that sees one key has P = 1 whatever the score: dS is 0, where the difference of dO.v and Delta would leave their roundings.  A
// loop of its own, as hardly any tile has such a query (inside the scores' loop packed documents trained 3 % slower); but beside a bias, where
// that loop is the longest, one loop more does not fit the instruction cache (16K tokens: 5.90 ms, against 5.66 inside).
__device__ __forceinline__ void drop_singles(uint32_t (&st)[32], const uint16_t *win) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(win + i);
        if (w & 0x80) st[i] = 0;
        if (w & 0x800000) st[i + 1] = 0;
    }
}

// Where 32 columns from `col` on of a key row's dK (which 0) or dV (which 1) go: the result, or a part's fp32 sums
template <bool kSmall, int R>
__device__ __forceinline__ void store_kv(const MaskedBwdParams<R> &p, const MbItem &it, int which, int row, int col, const uint32_t (&rr)[32]) {
    const int key = it.n * kT + row;
    if (key >= p.S) return;
    const size_t off = (((size_t)it.bl * p.S + key) * p.Hkv_l + it.hkv) * p.Dg + col;
    if (kSmall && p.parts > 1) {
        float *to = p.kv_part + ((size_t)(it.r * p.parts + it.part) * 2 + which) * p.kv_elems + off;
#pragma unroll
        for (int i = 0; i < 32; i += 4)
            if (col + i < p.Dg) *reinterpret_cast<uint4 *>(to + i) = make_uint4(rr[i], rr[i + 1], rr[i + 2], rr[i + 3]);
        return;
    }
    __nv_bfloat16 *to = (which ? p.dv[it.r] : p.dk[it.r]) + off;
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        uint4 o4;
        o4.x = pack_bf16x2(__uint_as_float(rr[i + 0]), __uint_as_float(rr[i + 1]));
        o4.y = pack_bf16x2(__uint_as_float(rr[i + 2]), __uint_as_float(rr[i + 3]));
        o4.z = pack_bf16x2(__uint_as_float(rr[i + 4]), __uint_as_float(rr[i + 5]));
        o4.w = pack_bf16x2(__uint_as_float(rr[i + 6]), __uint_as_float(rr[i + 7]));
        if (col + i < p.Dg) *reinterpret_cast<uint4 *>(to + i) = o4;
    }
}
// dK and dV of a key tile that no query sees: a quarter g of the compute warps takes 32 of the 128 columns of its row.  Where a sequence is
// one key tile its queries see nothing either, and dQ is zero.
template <bool kSmall, int R>
__device__ __forceinline__ void store_zeros(const MaskedBwdParams<R> &p, const MbItem &it, int g, int row) {
    const uint32_t zeros[32] = {};
    for (int which = 0; which < 2; ++which)
        if (32 * g < p.Dg) store_kv<kSmall>(p, it, which, row, 32 * g, zeros);
    if (kSmall && p.direct && row < p.S)
        for (int h = mb_first_head<kSmall>(p, it); h < mb_first_head<kSmall>(p, it) + mb_heads<kSmall>(p, it); ++h)
            for (int c = 32 * g; c < min(32 * g + 32, p.Dg); c += 8)
                *reinterpret_cast<uint4 *>(p.dq[it.r] + (((size_t)it.bl * p.S + row) * p.Hq_l + h) * p.Dg + c) = make_uint4(0, 0, 0, 0);
}

#include "attn_masked_bwd_d64.cuh"
#include "attn_masked_bwd_d128.cuh"

// In front of the products: Delta[bl][h][s] of every row (16 lanes a row, eight features a lane), and the dQ accumulator set to zero.
//
// Delta is dO.O, but O comes rounded to bf16 and from rounded P: an error of some 2^-9 |dO||O| against dO.v - Delta, which is of the size
// |dO||v|.  O is smaller by the root of the number of keys that count: over many rows dQ and dK are off by 0.37 % (2-norm) at two keys
// a row, 0.26 % at eight and 0.25 % from there on (dS and the result rounded), but a few rows by themselves, as of a sequence of two to six
// tokens, by 1.4 %.  Rows of up to kExactKeys keys therefore take Delta = sum_j P_ij dO_i.v_j from the scores, in fp32 (with 32 keys instead of
// eight, 8K tokens in documents of 40 trained in 515 us instead of 423; without any 389).
// One launch for every rank: blockIdx.y = rank.
constexpr int kExactKeys = 8;
constexpr int kKeysAtOnce = 4;       // keys in flight: 128 bytes a lane

template <int R>
struct PrepareParams {
    const __nv_bfloat16 *q[R], *k[R], *v[R], *o[R], *dout[R];
    const float *lse[R];
    float *delta[R], *acc[R];
    ScoreArgs score;
    int K, Bl, S, H, Hkv, D, causal, n_tiles, zero;
    float scale_log2;
    long long rows;
    FastDiv div_h, div_s, div_q_per_kv;
};

__device__ __forceinline__ float dot8(const uint4 &a, const uint4 &b) {
    const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
    float acc = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        acc = fmaf(__uint_as_float(av[i] << 16), __uint_as_float(bv[i] << 16), acc);
        acc = fmaf(__uint_as_float(av[i] & 0xffff0000u), __uint_as_float(bv[i] & 0xffff0000u), acc);
    }
    return acc;
}

template <int R>
__global__ void __launch_bounds__(256) mb_prepare_kernel(const __grid_constant__ PrepareParams<R> p) {
    const int part = threadIdx.x % 16, r = blockIdx.y;
    const uint32_t group = 0xffffu << (threadIdx.x & 16);        // the lanes of this row
    const long long row = (long long)blockIdx.x * 16 + threadIdx.x / 16;
    allow_next_kernel();
    if (row >= p.rows) return;                                   // (all lanes of the row)
    const bool mine = part * 8 < p.D;
    const uint4 none = make_uint4(0, 0, 0, 0);
    const size_t at = (size_t)row * p.D + part * 8;
    const uint4 up = mine ? *reinterpret_cast<const uint4 *>(p.dout[r] + at) : none;
    const uint4 o = mine ? *reinterpret_cast<const uint4 *>(p.o[r] + at) : none;
    if (p.zero && mine) {
        float4 *to = reinterpret_cast<float4 *>(p.acc[r] + at);
        to[0] = to[1] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const long long sb = p.rows <= 0x7fffffffll ? (long long)fdiv((uint32_t)row, p.div_h) : row / p.H;
    const int h = (int)(row - sb * p.H), bl = (int)fdiv((uint32_t)sb, p.div_s), s = (int)sb - bl * p.S;
    int lo = 0, hi = p.causal ? s + 1 : p.S;
    if (p.score.range) {
        const int2 range = __ldg(p.score.range + ((size_t)(r / p.K * p.Bl + bl) * p.n_tiles * kT + s));
        lo = max(range.x, 0);                     // (whatever the buffer holds, nothing outside of the sequence is read)
        hi = min(range.y, p.S);
    }
    float *delta = p.delta[r] + ((size_t)bl * p.H + h) * p.S + s;
    if (hi - lo > kExactKeys) {
        float acc = dot8(o, up);
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) acc += __shfl_xor_sync(group, acc, off);
        if (part == 0) *delta = acc;
        return;
    }
    const uint4 q = mine ? *reinterpret_cast<const uint4 *>(p.q[r] + at) : none;
    const float lse = seen_lse(p.lse[r][((size_t)bl * p.H + h) * p.S + s]);
    const float slope = p.score.slopes ? __ldg(p.score.slopes + r % p.K * p.H + h) * 1.4426950408889634f : 0.f;
    const size_t step = (size_t)p.Hkv * p.D, first = ((size_t)bl * p.S * p.Hkv + (int)fdiv((uint32_t)h, p.div_q_per_kv)) * p.D + part * 8;
    const bool upper = part & 8;
    float sum = 0.f;                     // of the keys so far, in every lane
#pragma unroll 1
    for (int j = lo; j < hi; j += kKeysAtOnce) {
        uint4 kk[kKeysAtOnce], vv[kKeysAtOnce];
#pragma unroll
        for (int i = 0; i < kKeysAtOnce; ++i) {
            const bool there = mine && j + i < hi;
            kk[i] = there ? *reinterpret_cast<const uint4 *>(p.k[r] + first + (j + i) * step) : none;
            vv[i] = there ? *reinterpret_cast<const uint4 *>(p.v[r] + first + (j + i) * step) : none;
        }
#pragma unroll
        for (int i = 0; i < kKeysAtOnce; ++i) {
            // q.k to the lower eight lanes, dO.v to the upper eight
            const float a = dot8(q, kk[i]), b = dot8(up, vv[i]);
            float mine2 = upper ? b : a;
            mine2 += __shfl_xor_sync(group, upper ? a : b, 8);
#pragma unroll
            for (int off = 4; off > 0; off >>= 1) mine2 += __shfl_xor_sync(group, mine2, off);
            const float other = __shfl_xor_sync(group, mine2, 8), raw = upper ? other : mine2, dp = upper ? mine2 : other;
            float z = p.score.cap_out > 0.f ? capped_any(raw, p.score) : raw * p.scale_log2;
            z -= slope * fabsf((float)(s - (j + i)));
            if (j + i < hi) sum = fmaf(exp2_approx(z - lse), dp, sum);
        }
    }
    if (part == 0) *delta = sum;
}

// Behind the products: dQ's accumulator to bf16 (n_q vectors of eight a rank) and the parts of dK and dV added up in order (n_kv vectors of
// each; none where the heads are not divided).  blockIdx.y = rank.
template <int R>
struct FinishParams {
    const float *acc[R];
    __nv_bfloat16 *dq[R], *dk[R], *dv[R];
    const float *kv_part;
    long long n_q, n_kv;
    int parts;
};
template <int R>
__global__ void __launch_bounds__(256) mb_finish_kernel(const __grid_constant__ FinishParams<R> p) {
    const int r = blockIdx.y;
    long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    wait_previous_kernel();
    float4 a, b;
    __nv_bfloat16 *to;
    if (i < p.n_q) {
        const float4 *from = reinterpret_cast<const float4 *>(p.acc[r]) + 2 * i;
        a = from[0];
        b = from[1];
        to = p.dq[r] + 8 * i;
    } else {
        i -= p.n_q;
        const int which = i >= p.n_kv;
        if (which) i -= p.n_kv;
        if (i >= p.n_kv) return;
        const float4 *from = reinterpret_cast<const float4 *>(p.kv_part) + ((long long)r * p.parts * 2 + which) * 2 * p.n_kv + 2 * i;
        a = from[0];
        b = from[1];
        for (int k = 1; k < p.parts; ++k) {
            from += 4 * p.n_kv;
            const float4 c = from[0], d = from[1];
            a.x += c.x; a.y += c.y; a.z += c.z; a.w += c.w;
            b.x += d.x; b.y += d.y; b.z += d.z; b.w += d.w;
        }
        to = (which ? p.dv[r] : p.dk[r]) + 8 * i;
    }
    *reinterpret_cast<uint4 *>(to) = make_uint4(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y), pack_bf16x2(b.z, b.w));
}

// Query heads of a key head that one work item takes.  All of them keep dK and dV in the tensor memory; but where the items are few, the
// longest one (a key tile that all query tiles see) is much of the whole: they are divided until it is below 0.6 of an SM's share, and the
// parts of dK and dV are added up behind (3001 tokens, 12/4 heads of 64, capped and biased: 185 us,
// 160 with the work divided).
int mb_part_heads(const basp_plan *p) {
    const int q_per_kv = p->Hq_l / p->Hkv_l;
    const double n = (p->S + kT - 1) / kT, pairs = p->causal ? n * (n + 1) / 2 : n * n;
    const double share = pairs * p->N * p->Bl * p->Hkv_l * q_per_kv / 148.0;
    int heads = q_per_kv;
    while (heads > 1 && heads * n > 0.6 * share) --heads;
    return heads;
}
int mb_parts(const basp_plan *p) {
    const int heads = mb_part_heads(p), q_per_kv = p->Hq_l / p->Hkv_l;
    return (q_per_kv + heads - 1) / heads;
}
size_t mb_kv_elems(const basp_plan *p) { return (size_t)p->Bl * p->S * p->Hkv_l * p->D; }
// accumulator and Delta of every rank, and the parts of dK and dV
size_t mb_workspace_bytes(const basp_plan *p) {
    const int parts = mb_parts(p);
    return (size_t)p->N * (bwd_acc_bytes(p) + bwd_delta_bytes(p) + (parts > 1 ? parts * 2 * mb_kv_elems(p) * sizeof(float) : 0));
}

template <int R>
int mb_run(const basp_plan *pl, const basp_score *score, const void *const *q, const void *const *k, const void *const *v,
           const void *const *o, const void *const *dout, const float *const *lse, void *const *dq, void *const *dk, void *const *dv,
           char *ws, float scale, cudaStream_t st) {
    MaskedBwdParams<R> prm;
    BASP_TRY(basp_score_args(pl, score, scale, &prm.score));
    const uint64_t rows = (uint64_t)pl->Bl * pl->S;
    const size_t acc_b = bwd_acc_bytes(pl), del_b = bwd_delta_bytes(pl);
    PrepareParams<R> pre;
    FinishParams<R> fin;
    for (int r = 0; r < pl->N; ++r) {
        BASP_TRY(tmap::encode_rows_heads_d(&prm.q[r], q[r], rows, pl->Hq_l, pl->D, kT));
        BASP_TRY(tmap::encode_rows_heads_d(&prm.k[r], k[r], rows, pl->Hkv_l, pl->D, kT));
        BASP_TRY(tmap::encode_rows_heads_d(&prm.v[r], v[r], rows, pl->Hkv_l, pl->D, kT));
        BASP_TRY(tmap::encode_rows_heads_d(&prm.dout[r], dout[r], rows, pl->Hq_l, pl->D, kT));
        float *acc = reinterpret_cast<float *>(ws + (size_t)r * acc_b);
        float *delta = reinterpret_cast<float *>(ws + (size_t)pl->N * acc_b + (size_t)r * del_b);
        if (pl->D <= 64) BASP_TRY(tmap::encode_f32_rows_heads_d(&prm.dq_acc[r], acc, rows, pl->Hq_l, pl->D, 32));
        prm.dq_accp[r] = acc;
        prm.lse[r] = lse[r];
        prm.delta[r] = delta;
        prm.dk[r] = (__nv_bfloat16 *)dk[r];
        prm.dv[r] = (__nv_bfloat16 *)dv[r];
        pre.q[r] = (const __nv_bfloat16 *)q[r];
        pre.k[r] = (const __nv_bfloat16 *)k[r];
        pre.v[r] = (const __nv_bfloat16 *)v[r];
        pre.o[r] = (const __nv_bfloat16 *)o[r];
        pre.dout[r] = (const __nv_bfloat16 *)dout[r];
        pre.lse[r] = lse[r];
        pre.delta[r] = delta;
        pre.acc[r] = acc;
        prm.dq[r] = (__nv_bfloat16 *)dq[r];
        fin.acc[r] = acc;
        fin.dq[r] = (__nv_bfloat16 *)dq[r];
        fin.dk[r] = (__nv_bfloat16 *)dk[r];
        fin.dv[r] = (__nv_bfloat16 *)dv[r];
    }
    prm.parts = mb_parts(pl);
    prm.part_heads = mb_part_heads(pl);
    prm.kv_part = reinterpret_cast<float *>(ws + (size_t)pl->N * (acc_b + del_b));
    prm.kv_elems = mb_kv_elems(pl);
    prm.direct = pl->S <= kT;            // one key tile: nothing to add up, dQ leaves as bf16
    prm.K = pl->K; prm.Bl = pl->Bl; prm.S = pl->S; prm.Hq_l = pl->Hq_l; prm.Hkv_l = pl->Hkv_l;
    prm.q_per_kv = pl->Hq_l / pl->Hkv_l; prm.causal = pl->causal;
    prm.n_tiles = (pl->S + kT - 1) / kT;
    prm.Dg = pl->D;
    const long long per = (long long)pl->K * pl->Hkv_l * prm.parts, total = (long long)pl->B * prm.n_tiles * per;
    const long long q_rows = (long long)rows * pl->Hq_l;
    fin.n_q = prm.direct ? 0 : (long long)(acc_b / sizeof(float) / 8);
    fin.n_kv = prm.parts > 1 ? (long long)(prm.kv_elems / 8) : 0;
    fin.kv_part = prm.kv_part;
    fin.parts = prm.parts;
    const long long n_fin = fin.n_q + 2 * fin.n_kv;
    if (total >= (1ll << 31) - 4096 || rows >= (1ull << 31) || q_rows >= (1ll << 35) || n_fin >= (1ll << 39)) return BASP_ERR_UNSUPPORTED;   // 31-bit items, rows, blocks
    prm.total = (int)total;
    prm.scale = scale;
    prm.scale_log2 = scale * 1.4426950408889634f;
    prm.status = basp_status_device_ptr();
    if (!prm.status) return BASP_ERR_CUDA;
    prm.div_items = make_fastdiv((uint32_t)per);
    prm.div_parts = make_fastdiv((uint32_t)prm.parts);
    prm.div_hkv_l = make_fastdiv((uint32_t)pl->Hkv_l);
    prm.div_B = make_fastdiv((uint32_t)pl->B);
    prm.div_bl = make_fastdiv((uint32_t)pl->Bl);
    int sms = 0;
    BASP_TRY(sm_count(&sms));
    const int grid = (int)(total < sms ? total : sms);

    pre.score = prm.score;
    pre.K = pl->K; pre.Bl = pl->Bl; pre.S = pl->S; pre.H = pl->Hq_l; pre.Hkv = pl->Hkv_l; pre.D = pl->D;
    pre.causal = pl->causal;
    pre.n_tiles = prm.n_tiles;
    pre.zero = !prm.direct;
    pre.scale_log2 = prm.scale_log2;
    pre.rows = q_rows;
    pre.div_h = make_fastdiv((uint32_t)pl->Hq_l);
    pre.div_s = make_fastdiv((uint32_t)pl->S);
    pre.div_q_per_kv = make_fastdiv((uint32_t)prm.q_per_kv);
    mb_prepare_kernel<R><<<dim3((unsigned)((q_rows + 15) / 16), (unsigned)pl->N), 256, 0, st>>>(pre);
    BASP_CUDA_TRY(cudaGetLastError());
    BASP_TRY(dispatch_score(prm.score.cap_out > 0.f, prm.score.slopes != nullptr, [&](auto cap, auto bias) -> int {
        constexpr bool kCap = decltype(cap)::value, kBias = decltype(bias)::value;
        // tiles, row statistics, windows, edge flags, barriers
        constexpr int smem128 = 7 * kT * 128 * 2 + 4 * kT * 4 + 2 * kT * 2 + 2 * 4 + (int)sizeof(BwdBars);
        constexpr int smem64 = (2 + 2 * 3) * kT * 64 * 2 + 4 * 16384 + 2 * 3 * kT * 4 + 3 * kT * 2 + 4 * 4 + (int)sizeof(BwdBars);
        const auto go = [&](auto small) -> int {
            constexpr bool kSmall = decltype(small)::value;
            if (pl->D > 64) {
                BASP_TRY((allow_smem<attn_masked_bwd_d128_kernel<R, kCap, kBias, kSmall>, smem128>()));
                BASP_CUDA_TRY(launch_early_smem(attn_masked_bwd_d128_kernel<R, kCap, kBias, kSmall>, dim3(grid), kBwdThreads, smem128, st, prm));
            } else {
                BASP_TRY((allow_smem<attn_masked_bwd_d64_kernel<R, kCap, kBias, kSmall>, smem64>()));
                BASP_CUDA_TRY(launch_early_smem(attn_masked_bwd_d64_kernel<R, kCap, kBias, kSmall>, dim3(grid), kBwdThreads, smem64, st, prm));
            }
            return BASP_OK;
        };
        return prm.parts > 1 || prm.direct ? go(std::true_type{}) : go(std::false_type{});
    }));
    if (n_fin > 0)
        BASP_CUDA_TRY(launch_early(mb_finish_kernel<R>, dim3((unsigned)((n_fin + 255) / 256), (unsigned)pl->N), 256, st, fin));
    basp_count_launch(n_fin > 0 ? 3 : 2);
    return BASP_OK;
}

}  // namespace

extern "C" size_t basp_attn_masked_bwd_workspace_bytes(const basp_plan *p) { return p ? mb_workspace_bytes(p) : 0; }

int basp_attn_masked_bwd_check(const basp_plan *pl, const basp_score *score, const void *const *q_head, const void *const *k_head,
                               const void *const *v_head, const void *const *o_head, const void *const *do_head,
                               const float *const *lse_shards, void *const *dq_head, void *const *dk_head, void *const *dv_head,
                               void *workspace, size_t workspace_bytes, float softmax_scale) {
    if (!pl || !score || !q_head || !k_head || !v_head || !o_head || !do_head || !lse_shards || !dq_head || !dk_head || !dv_head)
        return BASP_ERR_NULL;
    if (!scale_ok(softmax_scale)) return BASP_ERR_INVALID;
    if (pl->D < 16 || pl->D > 128 || pl->D % 16 != 0) return BASP_ERR_UNSUPPORTED;
    SpanSet spans;
    const size_t rows = (size_t)pl->Bl * pl->S, q_bytes = rows * pl->Hq_l * pl->D * 2, k_bytes = rows * pl->Hkv_l * pl->D * 2;
    for (int r = 0; r < pl->N; ++r) {
        const void *q_like[3] = {q_head[r], o_head[r], do_head[r]}, *k_like[2] = {k_head[r], v_head[r]};
        for (const void *t : q_like) BASP_TRY(spans.add_in(t, q_bytes));
        for (const void *t : k_like) BASP_TRY(spans.add_in(t, k_bytes));
        BASP_TRY(spans.add_in(lse_shards[r], rows * pl->Hq_l * 4));
        BASP_TRY(spans.add_out(dq_head[r], q_bytes));
        BASP_TRY(spans.add_out(dk_head[r], k_bytes));
        BASP_TRY(spans.add_out(dv_head[r], k_bytes));
    }
    if (score->slopes) BASP_TRY(spans.add_in(score->slopes, (size_t)pl->Hq * 4, 4));
    if (score->mask) BASP_TRY(spans.add_in(score->mask, basp_mask_bytes(pl)));
    BASP_TRY(spans.add_out(workspace, mb_workspace_bytes(pl)));
    if (workspace_bytes < mb_workspace_bytes(pl)) return BASP_ERR_WORKSPACE;
    BASP_TRY(spans.overlaps());
    ScoreArgs args;
    return basp_score_args(pl, score, resolved_scale(pl, softmax_scale), &args);
}

extern "C" int basp_attn_masked_bwd(const basp_plan *pl, const basp_score *score, const void *const *q_head, const void *const *k_head,
                                    const void *const *v_head, const void *const *o_head, const void *const *do_head,
                                    const float *const *lse_shards, void *const *dq_head, void *const *dk_head, void *const *dv_head,
                                    void *workspace, size_t workspace_bytes, float softmax_scale, void *stream) {
    BASP_TRY(basp_attn_masked_bwd_check(pl, score, q_head, k_head, v_head, o_head, do_head, lse_shards, dq_head, dk_head, dv_head, workspace,
                                        workspace_bytes, softmax_scale));
    const float scale = resolved_scale(pl, softmax_scale);
    return pl->N <= 8 ? mb_run<8>(pl, score, q_head, k_head, v_head, o_head, do_head, lse_shards, dq_head, dk_head, dv_head,
                                  (char *)workspace, scale, (cudaStream_t)stream)
                      : mb_run<BASP_MAX_RANKS>(pl, score, q_head, k_head, v_head, o_head, do_head, lse_shards, dq_head, dk_head, dv_head,
                                               (char *)workspace, scale, (cudaStream_t)stream);
}
