// Root-mean-square norm of every query and key head with the rotary position embedding in the same pass, over all
// ranks' sequence shards, and its backward pass.  For one head vector x of D features at position pos:
//
//   r = (mean x^2 + eps)^(-1/2),   z = r x w,   y = R(pos) z        (rotate-half: feature j < D/2 pairs with j + D/2)
//   backward:  u = R(pos)^T dy,   dw += r x u  (over all tokens and heads),   dx = r w u - x r^3 (x . w u) / D
//
// HBM-bound: 2 bytes read and 2 written per element forward, 4 read and 2 written backward.  All loads and stores are 16 bytes
// (eight features); the arithmetic is fp32 on packed pairs.  A token's cos and sin are fetched once for the heads of a work item.
// What the kernels wait for is memory latency, so they are laid out by the bytes in flight per SM that the registers allow:
//   forward   a lane holds eight features, D/8 lanes a vector, a warp 32 / (D/8) neighbouring heads of one token (of 512 bytes at
//             D = 128); the rotation's partner comes by shuffle.  80 registers, three blocks of 256 threads per SM.
//             2 x 8K tokens, 64 heads of 128: 97 us (5.6 TB/s); with the backward's layout a tenth more.
//   backward  a lane holds eight features and their eight partners, so D/16 lanes a vector and no shuffle but the sums; the
//             vectors of a warp are neighbouring tokens.  128 registers, two blocks per SM.
//             128K tokens, 40 heads of 128: 714 us (5.7 TB/s); with the forward's layout 727 us.
// The blocks are divided between Q and K by their heads (fill), which is even where both have as many; with fewer key heads K's blocks
// go on after Q's are done (128K tokens, 32 + 8 heads forward: 587 us, 4.6 TB/s).
#include <cuda_bf16.h>

#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"
#include "spans.h"

namespace {

using namespace ptx;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kFwdBlocks = 3, kBwdBlocks = 2;      // per SM
constexpr int kFwdUnroll = 4, kBwdUnroll = 2;      // vectors in flight per lane: 64 and 128 bytes

// R: room for ranks (8 or BASP_MAX_RANKS; a launch takes longer the larger its parameters)
template <int R>
struct HeadSet {               // one of the two tensors (Q or K) of all ranks
    const __nv_bfloat16 *x[R];
    const __nv_bfloat16 *dy[R];                   // backward only
    __nv_bfloat16 *out[R];                        // y, or dx
    const __nv_bfloat16 *w;
    uint32_t heads, chunks;    // heads per token, work items per token tile
    uint32_t chunk_heads;      // heads per work item
    uint32_t items;            // token tiles of all ranks x chunks
};

template <int R>
struct NormRopeParams {
    HeadSet<R> t[2];
    const float *cos, *sin;    // [D/2][S]
    float *partial;            // backward: [blocks][D] sums of dw
    float eps, inv_D;
    int D, S, T, T_last, K, Bl;
    uint32_t tiles, tile_tokens;   // token tiles per rank and their tokens
    int q_blocks;              // blocks that work on the first tensor (the others on the second)
};

__device__ __forceinline__ uint4 ld16(const __nv_bfloat16 *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void st16(__nv_bfloat16 *p, const uint4 &v) {
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" :: "l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Eight features as four packed pairs of fp32 (one instruction of the fp32 pipe works on a pair).
struct F8 { uint64_t p[4]; };
__device__ __forceinline__ F8 widen(const uint4 &v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    F8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.p[i] = pack_f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    return f;
}
__device__ __forceinline__ uint4 narrow(const F8 &f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpack_f2(f.p[i], lo, hi);
        w[i] = pack_bf16x2(lo, hi);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float sum2(uint64_t v) {
    float lo, hi;
    unpack_f2(v, lo, hi);
    return lo + hi;
}
// Sum over the N lanes that hold a vector, in all of them; `lane`: this one's place among them.  N up to 16, not only powers of two.
template <int N>
__device__ __forceinline__ float group_sum(float v, int lane) {
    if constexpr ((N & (N - 1)) == 0) {
#pragma unroll
        for (int o = N / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    } else {
#pragma unroll
        for (int o = N > 8 ? 8 : N > 4 ? 4 : 2; o > 0; o >>= 1) {
            const float far = __shfl_down_sync(0xffffffffu, v, o);
            if (lane + o < N) v += far;
        }
        return __shfl_sync(0xffffffffu, v, (threadIdx.x & 31) - lane);
    }
}

// A work item: some heads of a tile of neighbouring tokens of one rank.  The blocks of a tensor take its items in turn,
// so that at any time they read and write neighbouring memory.
struct Share {
    int which;
    uint32_t item, end, step;
};
template <int R>
__device__ __forceinline__ Share share_of(const NormRopeParams<R> &p) {
    Share o;
    o.which = (int)blockIdx.x >= p.q_blocks;
    o.item = o.which ? blockIdx.x - p.q_blocks : blockIdx.x;
    o.step = o.which ? gridDim.x - p.q_blocks : p.q_blocks;
    o.end = p.t[o.which].items;
    return o;
}

// The heads of an item and the tile's token number `token`.
struct Place {
    uint32_t rank;
    int count, pos;
    size_t off;                // the token's first element of the first of the heads in the rank's shard
    bool valid;                // the rank has such a token
};
template <int R>
__device__ __forceinline__ Place place_of(const NormRopeParams<R> &p, const HeadSet<R> &t, uint32_t item, uint32_t token) {
    Place o;
    const uint32_t tile = item / t.chunks, head = (item - tile * t.chunks) * t.chunk_heads;
    o.count = (int)min(t.chunk_heads, t.heads - head);
    o.rank = tile / p.tiles;
    const uint32_t row = (tile - o.rank * p.tiles) * p.tile_tokens + token, l = o.rank % p.K;
    const uint32_t Tr = (int)l == p.K - 1 ? p.T_last : p.T;
    o.pos = (int)(l * p.T + row % Tr);
    o.off = ((size_t)row * t.heads + head) * p.D;
    o.valid = row < p.Bl * Tr;
    return o;
}

// Eight features of a feature-major table at position pos.  The row pitch is kept from the optimiser: it would compute the eight
// offsets once for all items and spill them.
__device__ __forceinline__ F8 load_feature_major(const float *table, int S, int lane, int pos) {
    size_t pitch = (size_t)S;
    asm volatile("" : "+l"(pitch));
    const float *at = table + (size_t)(8 * lane) * pitch + pos;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __ldg(at + e * pitch);
    F8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.p[i] = pack_f2(v[2 * i], v[2 * i + 1]);
    return f;
}

// What a lane needs of another one: the eight features that the rotation pairs with its own, D/2 away.
__device__ __forceinline__ uint4 partner(const uint4 &v, int src) {
    return make_uint4(__shfl_sync(0xffffffffu, v.x, src), __shfl_sync(0xffffffffu, v.y, src), __shfl_sync(0xffffffffu, v.z, src),
                      __shfl_sync(0xffffffffu, v.w, src));
}

// N = D / 8 lanes hold a vector, a warp 32 / N neighbouring heads of its token.
template <int N, int R>
__global__ void __launch_bounds__(kThreads, kFwdBlocks) norm_rope_kernel(const __grid_constant__ NormRopeParams<R> p) {
    constexpr int kUnroll = kFwdUnroll, kVectors = 32 / N;
    const int warp_lane = threadIdx.x & 31, vec = warp_lane / N, lane = warp_lane - vec * N;
    const bool low = lane < N / 2, mine = vec < kVectors;
    const int other = low ? lane + N / 2 : lane - N / 2, src = vec * N + other;
    const Share share = share_of(p);
    const HeadSet<R> &t = p.t[share.which];
    for (uint32_t item = share.item; item < share.end; item += share.step) {
        const Place at = place_of(p, t, item, threadIdx.x / 32);
        if (!at.valid) continue;
        const __nv_bfloat16 *x = t.x[at.rank] + at.off + warp_lane * 8;
        __nv_bfloat16 *y = t.out[at.rank] + at.off + warp_lane * 8;
        const int count = at.count - vec;     // heads from this lane's first one on
        // weights folded into the rotation: y = r (x a + x' b) with x' the partner's and b's sign by the half
        F8 fa{}, fb{};
        for (int h = 0; h < at.count; h += kUnroll * kVectors) {
            uint4 raw[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                raw[u] = make_uint4(0, 0, 0, 0);
                if (mine && h + u * kVectors < count) raw[u] = ld16(x + u * (kVectors * N * 8));
            }
            if (h == 0 && mine) {                  // behind the first loads of x: their latencies overlap
                const F8 cv = load_feature_major(p.cos, p.S, low ? lane : other, at.pos);
                const F8 sv = load_feature_major(p.sin, p.S, low ? lane : other, at.pos);
                const F8 w = widen(ld16(t.w + 8 * lane)), wo = widen(ld16(t.w + 8 * other));
                const uint64_t sign = low ? pack_f2(-1.f, -1.f) : pack_f2(1.f, 1.f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    fa.p[e] = mul2(w.p[e], cv.p[e]);
                    fb.p[e] = mul2(mul2(wo.p[e], sv.p[e]), sign);
                }
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const F8 own = widen(raw[u]), far = widen(partner(raw[u], src));
                uint64_t sq = mul2(own.p[0], own.p[0]);
#pragma unroll
                for (int e = 1; e < 4; ++e) sq = fma2(own.p[e], own.p[e], sq);
                const float r = rsqrtf(fmaf(group_sum<N>(sum2(sq), lane), p.inv_D, p.eps));
                if (!mine || h + u * kVectors >= count) continue;
                const uint64_t r2 = pack_f2(r, r);
                F8 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o.p[e] = fma2(mul2(own.p[e], r2), fa.p[e], mul2(mul2(far.p[e], r2), fb.p[e]));
                st16(y + u * (kVectors * N * 8), narrow(o));
            }
            x += kUnroll * kVectors * N * 8;
            y += kUnroll * kVectors * N * 8;
        }
    }
}

// Backward: N = D / 16 lanes hold a vector, the vectors of a warp are one head of 32 / N neighbouring tokens.  A block keeps the dw sums
// of its features in registers, at the end adds its vectors together in shared memory and writes one partial row, in a fixed order
// (the result does not depend on timing).
template <int N, int R>
__global__ void __launch_bounds__(kThreads, kBwdBlocks) norm_rope_bwd_kernel(const __grid_constant__ NormRopeParams<R> p) {
    constexpr int kUnroll = kBwdUnroll, kVectors = 32 / N, half = 8 * N;
    __shared__ float part[kWarps * kVectors][16 * N];
    const int warp_lane = threadIdx.x & 31, vec = warp_lane / N, lane = warp_lane - vec * N;
    const Share share = share_of(p);
    const HeadSet<R> &t = p.t[share.which];
    const bool mine = vec < kVectors;
    const uint32_t token = threadIdx.x / 32 * kVectors + vec;
    allow_next_kernel();
    const uint64_t minus = pack_f2(-1.f, -1.f);
    F8 wl{}, wh{}, gl{}, gh{};
    if (mine) { wl = widen(ld16(t.w + 8 * lane)); wh = widen(ld16(t.w + half + 8 * lane)); }
    for (uint32_t item = share.item; item < share.end; item += share.step) {
        const Place at = place_of(p, t, item, token);
        const bool active = at.valid && mine;
        const __nv_bfloat16 *x = t.x[at.rank] + at.off + 8 * lane, *dy = t.dy[at.rank] + at.off + 8 * lane;
        __nv_bfloat16 *dx = t.out[at.rank] + at.off + 8 * lane;
        F8 cv{}, sv{};
        for (int h = 0; h < at.count; h += kUnroll) {
            uint4 rx[kUnroll][2], ry[kUnroll][2];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                rx[u][0] = rx[u][1] = ry[u][0] = ry[u][1] = make_uint4(0, 0, 0, 0);
                if (active && h + u < at.count) {
                    const size_t o = (size_t)(h + u) * p.D;
                    rx[u][0] = ld16(x + o); rx[u][1] = ld16(x + o + half);
                    ry[u][0] = ld16(dy + o); ry[u][1] = ld16(dy + o + half);
                }
            }
            if (h == 0 && active) {                // behind the first loads: their latencies overlap
                cv = load_feature_major(p.cos, p.S, lane, at.pos);
                sv = load_feature_major(p.sin, p.S, lane, at.pos);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const F8 xl = widen(rx[u][0]), xh = widen(rx[u][1]);
                F8 ul = widen(ry[u][0]), uh = widen(ry[u][1]);
                uint64_t sq = 0, dot = 0;          // pairs of zeros
#pragma unroll
                for (int e = 0; e < 4; ++e) {      // u = R^T dy
                    const uint64_t l = fma2(ul.p[e], cv.p[e], mul2(uh.p[e], sv.p[e]));
                    const uint64_t g = fma2(uh.p[e], cv.p[e], mul2(mul2(ul.p[e], minus), sv.p[e]));
                    ul.p[e] = l; uh.p[e] = g;
                    sq = fma2(xl.p[e], xl.p[e], fma2(xh.p[e], xh.p[e], sq));
                    dot = fma2(xl.p[e], mul2(l, wl.p[e]), fma2(xh.p[e], mul2(g, wh.p[e]), dot));
                }
                const float s1 = group_sum<N>(sum2(sq), lane), s2 = group_sum<N>(sum2(dot), lane);
                const float r = rsqrtf(fmaf(s1, p.inv_D, p.eps));
                if (!active || h + u >= at.count) continue;
                const float k = -(r * s2 * p.inv_D) * r * r;     // in this order: r^3 alone leaves fp32 for zeros and an eps below 1e-25
                const uint64_t r2 = pack_f2(r, r), k2 = pack_f2(k, k);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t l = mul2(ul.p[e], r2), g = mul2(uh.p[e], r2);
                    gl.p[e] = fma2(xl.p[e], l, gl.p[e]);
                    gh.p[e] = fma2(xh.p[e], g, gh.p[e]);
                    ul.p[e] = fma2(wl.p[e], l, mul2(xl.p[e], k2));
                    uh.p[e] = fma2(wh.p[e], g, mul2(xh.p[e], k2));
                }
                const size_t o = (size_t)(h + u) * p.D;
                st16(dx + o, narrow(ul));
                st16(dx + o + half, narrow(uh));
            }
        }
    }
    if (mine) {
        float *dst = part[token] + 8 * lane;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            unpack_f2(gl.p[e], dst[2 * e], dst[2 * e + 1]);
            unpack_f2(gh.p[e], dst[half + 2 * e], dst[half + 2 * e + 1]);
        }
    }
    __syncthreads();
    if (threadIdx.x < 16 * N) {
        float s = 0.f;
#pragma unroll 16
        for (int k = 0; k < kWarps * kVectors; ++k) s += part[k][threadIdx.x];
        p.partial[(size_t)blockIdx.x * p.D + threadIdx.x] = s;
    }
}

// dw of both tensors from the blocks' partial rows: a block takes eight features of one tensor, 32 threads a feature.
__global__ void __launch_bounds__(256) dw_kernel(const float *partial, int D, int q_blocks, int blocks, float *dw_q, float *dw_k) {
    __shared__ float part[32][9];
    const int f = threadIdx.x % 8, i = threadIdx.x / 8, col = blockIdx.x * 8 + f;
    const int b0 = blockIdx.y ? q_blocks : 0, b1 = blockIdx.y ? blocks : q_blocks;
    float s = 0.f;
    wait_previous_kernel();
#pragma unroll 8
    for (int b = b0 + i; b < b1; b += 32) s += partial[(size_t)b * D + col];
    part[i][f] = s;
    __syncthreads();
    if (i == 0) {
        for (int k = 1; k < 32; ++k) s += part[k][f];
        (blockIdx.y ? dw_k : dw_q)[col] = s;
    }
}

// What both directions share: the geometry and the split of the work over one wave of blocks, in items of tile_tokens tokens and some
// of their heads (`batch`: the heads of a token that are in flight).
template <int R>
int fill(const basp_plan *p, const void *w_q, const void *w_k, const float *cos, const float *sin, float eps, int tile_tokens,
         int batch, int wave, NormRopeParams<R> *prm, int *blocks) {
    const long long rows = (long long)p->Bl * p->T, tiles = (rows + tile_tokens - 1) / tile_tokens;
    if (tiles * tile_tokens >= (1ll << 31) || tiles * p->N * p->Hq >= (1ll << 31)) return BASP_ERR_UNSUPPORTED;     // 31-bit rows, items
    prm->cos = cos; prm->sin = sin; prm->eps = eps; prm->inv_D = 1.0f / (float)p->D;
    prm->D = p->D; prm->S = p->S; prm->T = p->T; prm->T_last = p->T_last; prm->K = p->K; prm->Bl = p->Bl;
    prm->tiles = (uint32_t)tiles; prm->tile_tokens = (uint32_t)tile_tokens;
    prm->t[0].w = (const __nv_bfloat16 *)w_q; prm->t[0].heads = p->Hq;
    prm->t[1].w = (const __nv_bfloat16 *)w_k; prm->t[1].heads = p->Hkv;
    // blocks in proportion to the heads, at least one per tensor
    const long long units = tiles * p->N;
    int q = (wave * p->Hq + (p->Hq + p->Hkv) / 2) / (p->Hq + p->Hkv);
    q = q < 1 ? 1 : (q > wave - 1 ? wave - 1 : q);
    for (HeadSet<R> &t : prm->t) {
        // A tile's heads in n items: few, and a token's cos and sin are fetched for more of them; many, and the last round of items
        // over the blocks is short.  An item costs its batches of heads and a start of three quarters of a batch
        const int blocks_of = &t == &prm->t[0] ? q : wave - q;
        double best = 1e30;
        for (uint32_t n = 1; n <= t.heads && n <= 32; ++n) {
            const uint32_t heads = (t.heads + n - 1) / n;
            const double cost = (double)((units * n + blocks_of - 1) / blocks_of) * ((heads + batch - 1) / batch + 0.75);
            if (cost < best) { best = cost; t.chunk_heads = heads; }
        }
        t.chunks = (t.heads + t.chunk_heads - 1) / t.chunk_heads;
        t.items = (uint32_t)(units * t.chunks);
    }
    if (q > (int)prm->t[0].items) q = (int)prm->t[0].items;                      // no block without an item
    const int k = wave - q < (int)prm->t[1].items ? wave - q : (int)prm->t[1].items;
    prm->q_blocks = q;
    *blocks = q + k;
    return BASP_OK;
}

int supported(const basp_plan *p, float eps) {
    if (p->D % 16 != 0 || p->D > 128) return BASP_ERR_UNSUPPORTED;
    return eps > 0.f && eps <= 3.0e38f ? BASP_OK : BASP_ERR_INVALID;
}

// Adds the shards of one tensor to the spans and the parameter block.
int add_shards(const basp_plan *p, SpanSet *s, int heads, const void *const *shards, bool out, int slot, const __nv_bfloat16 **to) {
    if (!shards) return BASP_ERR_NULL;
    for (int r = 0; r < p->N; ++r) {
        const size_t bytes = (size_t)p->Bl * basp_rank_tokens(p, r % p->K) * heads * p->D * 2;
        const int sl = slot < 0 ? -1 : slot * BASP_MAX_RANKS + r;
        BASP_TRY(out ? s->add_out(shards[r], bytes, 16, sl) : s->add_in(shards[r], bytes, 16, sl));
        to[r] = (const __nv_bfloat16 *)shards[r];
    }
    return BASP_OK;
}

int add_tables(const basp_plan *p, SpanSet *s, const void *w_q, const void *w_k, const float *cos, const float *sin) {
    const size_t table = (size_t)(p->D / 2) * p->S * 4;
    BASP_TRY(s->add_in(w_q, (size_t)p->D * 2));
    BASP_TRY(s->add_in(w_k, (size_t)p->D * 2));
    BASP_TRY(s->add_in(cos, table, 4));
    return s->add_in(sin, table, 4);
}

// f(the number as a type) for one of the listed numbers
template <int... kN, typename F>
int dispatch(int n, F &&f) {
    int rc = BASP_ERR_UNSUPPORTED;
    ((n == kN ? (void)(rc = f(std::integral_constant<int, kN>{})) : (void)0), ...);
    return rc;
}

template <int R>
int run_fwd(const basp_plan *p, const void *const *q_seq, const void *const *k_seq, const void *w_q, const void *w_k,
            const float *rope_cos, const float *rope_sin, float eps, void *const *q_out, void *const *k_out, void *stream) {
    NormRopeParams<R> prm;
    int blocks = 0;
    BASP_TRY(fill(p, w_q, w_k, rope_cos, rope_sin, eps, kWarps, kFwdUnroll * (32 / (p->D / 8)), 148 * kFwdBlocks, &prm, &blocks));
    SpanSet spans;
    BASP_TRY(add_tables(p, &spans, w_q, w_k, rope_cos, rope_sin));
    BASP_TRY(add_shards(p, &spans, p->Hq, q_seq, false, 0, prm.t[0].x));
    BASP_TRY(add_shards(p, &spans, p->Hkv, k_seq, false, 1, prm.t[1].x));
    BASP_TRY(add_shards(p, &spans, p->Hq, q_out, true, 0, const_cast<const __nv_bfloat16 **>(prm.t[0].out)));
    BASP_TRY(add_shards(p, &spans, p->Hkv, k_out, true, 1, const_cast<const __nv_bfloat16 **>(prm.t[1].out)));
    BASP_TRY(spans.overlaps());
    return dispatch<2, 4, 6, 8, 10, 12, 14, 16>(p->D / 8, [&](auto lanes) -> int {
        norm_rope_kernel<decltype(lanes)::value, R><<<blocks, kThreads, 0, (cudaStream_t)stream>>>(prm);
        BASP_CUDA_TRY(cudaGetLastError());
        basp_count_launch(1);
        return BASP_OK;
    });
}

size_t bwd_workspace_bytes(const basp_plan *p) { return (size_t)148 * kBwdBlocks * p->D * 4; }

template <int R>
int run_bwd(const basp_plan *p, const void *const *q_seq, const void *const *k_seq, const void *w_q, const void *w_k,
            const float *rope_cos, const float *rope_sin, float eps, const void *const *dq_out, const void *const *dk_out,
            void *const *dq_seq, void *const *dk_seq, float *dw_q, float *dw_k, void *workspace, size_t workspace_bytes,
            void *stream) {
    NormRopeParams<R> prm;
    int blocks = 0;
    BASP_TRY(fill(p, w_q, w_k, rope_cos, rope_sin, eps, kWarps * (32 / (p->D / 16)), kBwdUnroll, 148 * kBwdBlocks, &prm, &blocks));
    SpanSet spans;
    BASP_TRY(add_tables(p, &spans, w_q, w_k, rope_cos, rope_sin));
    BASP_TRY(add_shards(p, &spans, p->Hq, q_seq, false, -1, prm.t[0].x));
    BASP_TRY(add_shards(p, &spans, p->Hkv, k_seq, false, -1, prm.t[1].x));
    BASP_TRY(add_shards(p, &spans, p->Hq, dq_out, false, 0, prm.t[0].dy));
    BASP_TRY(add_shards(p, &spans, p->Hkv, dk_out, false, 1, prm.t[1].dy));
    BASP_TRY(add_shards(p, &spans, p->Hq, dq_seq, true, 0, const_cast<const __nv_bfloat16 **>(prm.t[0].out)));
    BASP_TRY(add_shards(p, &spans, p->Hkv, dk_seq, true, 1, const_cast<const __nv_bfloat16 **>(prm.t[1].out)));
    BASP_TRY(spans.add_out(dw_q, (size_t)p->D * 4, 4));
    BASP_TRY(spans.add_out(dw_k, (size_t)p->D * 4, 4));
    BASP_TRY(spans.add_out(workspace, bwd_workspace_bytes(p)));
    if (workspace_bytes < bwd_workspace_bytes(p)) return BASP_ERR_WORKSPACE;
    BASP_TRY(spans.overlaps());
    prm.partial = (float *)workspace;
    return dispatch<1, 2, 3, 4, 5, 6, 7, 8>(p->D / 16, [&](auto lanes) -> int {
        norm_rope_bwd_kernel<decltype(lanes)::value, R><<<blocks, kThreads, 0, (cudaStream_t)stream>>>(prm);
        BASP_CUDA_TRY(cudaGetLastError());
        BASP_CUDA_TRY(launch_early(dw_kernel, dim3(p->D / 8, 2), 256, (cudaStream_t)stream, (const float *)prm.partial, p->D, prm.q_blocks,
                                   blocks, dw_q, dw_k));
        basp_count_launch(2);
        return BASP_OK;
    });
}

}  // namespace

extern "C" int basp_qk_norm_rope(const basp_plan *p, const void *const *q_seq, const void *const *k_seq, const void *w_q,
                                 const void *w_k, const float *rope_cos, const float *rope_sin, float eps, void *const *q_out,
                                 void *const *k_out, void *stream) {
    if (!p) return BASP_ERR_NULL;
    BASP_TRY(supported(p, eps));
    return p->N <= 8 ? run_fwd<8>(p, q_seq, k_seq, w_q, w_k, rope_cos, rope_sin, eps, q_out, k_out, stream)
                     : run_fwd<BASP_MAX_RANKS>(p, q_seq, k_seq, w_q, w_k, rope_cos, rope_sin, eps, q_out, k_out, stream);
}

extern "C" size_t basp_qk_norm_rope_bwd_workspace_bytes(const basp_plan *p) { return p ? bwd_workspace_bytes(p) : 0; }

extern "C" int basp_qk_norm_rope_bwd(const basp_plan *p, const void *const *q_seq, const void *const *k_seq, const void *w_q,
                                     const void *w_k, const float *rope_cos, const float *rope_sin, float eps,
                                     const void *const *dq_out, const void *const *dk_out, void *const *dq_seq,
                                     void *const *dk_seq, float *dw_q, float *dw_k, void *workspace, size_t workspace_bytes,
                                     void *stream) {
    if (!p) return BASP_ERR_NULL;
    BASP_TRY(supported(p, eps));
    return p->N <= 8 ? run_bwd<8>(p, q_seq, k_seq, w_q, w_k, rope_cos, rope_sin, eps, dq_out, dk_out, dq_seq,
                                  dk_seq, dw_q, dw_k, workspace, workspace_bytes, stream)
                     : run_bwd<BASP_MAX_RANKS>(p, q_seq, k_seq, w_q, w_k, rope_cos, rope_sin, eps, dq_out, dk_out, dq_seq,
                                                  dk_seq, dw_q, dw_k, workspace, workspace_bytes, stream);
}
