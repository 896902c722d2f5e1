// Root-mean-square norm of every query and key head with the rotary position embedding in the same pass, over all
// ranks' sequence shards, and its backward pass.  For one head vector x of D features at position pos:
//
//   r = (mean x^2 + eps)^(-1/2),   z = r x w,   y = R(pos) z        (rotate-half: feature j < D/2 pairs with j + D/2)
//   backward:  u = R(pos)^T dy,   dw += r x u  (over all tokens and heads),   dx = r w u - x r^3 (x . w u) / D
//
// HBM-bound: 2 bytes read and 2 written per element forward, 4 read and 2 written backward, a few operations each.  A
// vector is held by D/16 neighbouring lanes, lane i with features 8i..8i+7 and the partners D/2 + 8i .. of the rotation,
// so that both halves of every pair are in one thread, every load and store is 16 bytes, and the sums of a vector cross
// at most three shuffles.  Where D/16 is no power of two the group of lanes is the next one and its last lanes idle.  A
// group owns one token and walks over heads: the token's cos and sin are fetched once for all of them.
#include <cuda_bf16.h>

#include "common.cuh"
#include "spans.h"

namespace {

constexpr int kThreads = 256;

struct HeadSet {               // one of the two tensors (Q or K) of all ranks
    const __nv_bfloat16 *x[BASP_MAX_RANKS];
    const __nv_bfloat16 *dy[BASP_MAX_RANKS];      // backward only
    __nv_bfloat16 *out[BASP_MAX_RANKS];           // y, or dx
    const __nv_bfloat16 *w;
    int heads, chunks;         // heads per token; head chunks per token tile
};

struct NormRopeParams {
    HeadSet t[2];
    const float *cos, *sin;    // [D/2][S]
    float *partial;            // backward: [blocks][D] sums of dw
    float eps, inv_D;
    int D, S, T, T_last, K, Bl, N;
    int chunk_heads;           // heads per chunk
    int tiles;                 // token tiles per rank
    int q_items, items;        // work items of the first tensor, and of both
    int q_blocks;              // backward: blocks that work on the first tensor (the others on the second)
    FastDiv div_T, div_T_last;
};

__device__ __forceinline__ uint4 ld16(const __nv_bfloat16 *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void st16(__nv_bfloat16 *p, const uint4 &v) {
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" :: "l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void widen(const uint4 &v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 narrow(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int L>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o, L);
    return v;
}

// The token tile and head chunk of a work item, and this thread's share of it.
struct Place {
    int rank, row, head_begin, head_end;
    bool active;               // this lane has features of a token of the tile
};

template <int L>
__device__ __forceinline__ Place place_of(const NormRopeParams &p, const HeadSet &t, int item, int group, int lane, int &pos) {
    constexpr int kTokens = kThreads / L;
    Place o;
    const int chunk = item % t.chunks, tile = item / t.chunks;
    o.rank = tile / p.tiles;
    const int l = o.rank % p.K;
    const bool last = l == p.K - 1;
    const int Tr = last ? p.T_last : p.T;
    o.row = (tile - o.rank * p.tiles) * kTokens + group;
    o.active = o.row < p.Bl * Tr && lane * 16 < p.D;
    const int bl = (int)fdiv((uint32_t)o.row, last ? p.div_T_last : p.div_T);
    pos = l * p.T + (o.row - bl * Tr);
    o.head_begin = chunk * p.chunk_heads;
    o.head_end = min(t.heads, o.head_begin + p.chunk_heads);
    return o;
}

// cos and sin of this thread's eight features at position pos (feature-major tables: the tile's tokens are neighbours).
__device__ __forceinline__ void load_angles(const NormRopeParams &p, int lane, int pos, float (&c)[8], float (&s)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const size_t at = (size_t)(8 * lane + e) * p.S + pos;
        c[e] = __ldg(p.cos + at);
        s[e] = __ldg(p.sin + at);
    }
}

template <int L>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const __grid_constant__ NormRopeParams p) {
    constexpr int kUnroll = 4;                     // heads in flight: 128 bytes per thread
    const int group = threadIdx.x / L, lane = threadIdx.x % L;
    int item = blockIdx.x;
    const HeadSet &t = p.t[item >= p.q_items];
    if (item >= p.q_items) item -= p.q_items;
    int pos;
    const Place at = place_of<L>(p, t, item, group, lane, pos);
    const int half = p.D / 2;
    const size_t row_elems = (size_t)t.heads * p.D;
    const size_t base = (size_t)at.row * row_elems + 8 * lane;
    const __nv_bfloat16 *x = t.x[at.rank] + base;
    __nv_bfloat16 *y = t.out[at.rank] + base;
    // weights folded into the rotation: y_lo = r (x_lo a - x_hi b), y_hi = r (x_hi c + x_lo d)
    float a[8], b[8], c[8], d[8];
    bool first = true;
    for (int h = at.head_begin; h < at.head_end; h += kUnroll) {
        uint4 lo[kUnroll], hi[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
            if (at.active && h + u < at.head_end) {
                lo[u] = ld16(x + (size_t)(h + u) * p.D);
                hi[u] = ld16(x + (size_t)(h + u) * p.D + half);
            }
        }
        if (first && at.active) {                  // behind the first loads of x: their latencies overlap
            float cv[8], sv[8], wl[8], wh[8];
            load_angles(p, lane, pos, cv, sv);
            widen(ld16(t.w + 8 * lane), wl);
            widen(ld16(t.w + half + 8 * lane), wh);
#pragma unroll
            for (int e = 0; e < 8; ++e) { a[e] = wl[e] * cv[e]; b[e] = wh[e] * sv[e]; c[e] = wh[e] * cv[e]; d[e] = wl[e] * sv[e]; }
        }
        first = false;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float xl[8], xh[8], sum = 0.f;
            widen(lo[u], xl);
            widen(hi[u], xh);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(xl[e], xl[e], fmaf(xh[e], xh[e], sum));
            const float r = rsqrtf(fmaf(group_sum<L>(sum), p.inv_D, p.eps));
            if (!at.active || h + u >= at.head_end) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float l = xl[e] * r, g = xh[e] * r;
                xl[e] = l * a[e] - g * b[e];
                xh[e] = g * c[e] + l * d[e];
            }
            st16(y + (size_t)(h + u) * p.D, narrow(xl));
            st16(y + (size_t)(h + u) * p.D + half, narrow(xh));
        }
    }
}

// Backward.  Persistent: a block walks over the items of ONE tensor and keeps the dw sums of its features in registers;
// at the end it adds its groups together in shared memory and writes one partial row, in a fixed order (the result does
// not depend on timing).
template <int L>
__global__ void __launch_bounds__(kThreads, 2) norm_rope_bwd_kernel(const __grid_constant__ NormRopeParams p) {
    constexpr int kUnroll = 2;
    __shared__ float part[kThreads / 32][128];
    const int group = threadIdx.x / L, lane = threadIdx.x % L;
    const int which = (int)blockIdx.x >= p.q_blocks;
    const HeadSet &t = p.t[which];
    const int n_items = which ? p.items - p.q_items : p.q_items;
    const int step = which ? (int)gridDim.x - p.q_blocks : p.q_blocks;
    const int half = p.D / 2;
    const size_t row_elems = (size_t)t.heads * p.D;
    float wl[8], wh[8], gl[8], gh[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) gl[e] = gh[e] = wl[e] = wh[e] = 0.f;
    if (lane * 16 < p.D) {
        widen(ld16(t.w + 8 * lane), wl);
        widen(ld16(t.w + half + 8 * lane), wh);
    }
    for (int item = (int)blockIdx.x - (which ? p.q_blocks : 0); item < n_items; item += step) {
        int pos;
        const Place at = place_of<L>(p, t, item, group, lane, pos);
        const size_t base = (size_t)at.row * row_elems + 8 * lane;
        const __nv_bfloat16 *x = t.x[at.rank] + base, *dy = t.dy[at.rank] + base;
        __nv_bfloat16 *dx = t.out[at.rank] + base;
        float cv[8], sv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) cv[e] = sv[e] = 0.f;
        if (at.active) load_angles(p, lane, pos, cv, sv);
        for (int h = at.head_begin; h < at.head_end; h += kUnroll) {
            uint4 rx[kUnroll][2], ry[kUnroll][2];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                rx[u][0] = rx[u][1] = ry[u][0] = ry[u][1] = make_uint4(0, 0, 0, 0);
                if (at.active && h + u < at.head_end) {
                    const size_t o = (size_t)(h + u) * p.D;
                    rx[u][0] = ld16(x + o); rx[u][1] = ld16(x + o + half);
                    ry[u][0] = ld16(dy + o); ry[u][1] = ld16(dy + o + half);
                }
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                float xl[8], xh[8], ul[8], uh[8], sq = 0.f, dot = 0.f;
                widen(rx[u][0], xl); widen(rx[u][1], xh);
                widen(ry[u][0], ul); widen(ry[u][1], uh);
#pragma unroll
                for (int e = 0; e < 8; ++e) {      // u = R^T dy
                    const float l = ul[e] * cv[e] + uh[e] * sv[e], g = uh[e] * cv[e] - ul[e] * sv[e];
                    ul[e] = l; uh[e] = g;
                    sq = fmaf(xl[e], xl[e], fmaf(xh[e], xh[e], sq));
                    dot = fmaf(xl[e], l * wl[e], fmaf(xh[e], g * wh[e], dot));
                }
                sq = group_sum<L>(sq);
                dot = group_sum<L>(dot);
                const float r = rsqrtf(fmaf(sq, p.inv_D, p.eps));
                const float k = r * r * r * dot * p.inv_D;
                if (!at.active || h + u >= at.head_end) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ul[e] *= r; uh[e] *= r;
                    gl[e] = fmaf(xl[e], ul[e], gl[e]);
                    gh[e] = fmaf(xh[e], uh[e], gh[e]);
                    ul[e] = ul[e] * wl[e] - xl[e] * k;
                    uh[e] = uh[e] * wh[e] - xh[e] * k;
                }
                const size_t o = (size_t)(h + u) * p.D;
                st16(dx + o, narrow(ul));
                st16(dx + o + half, narrow(uh));
            }
        }
    }
    // groups of a warp, then the warps
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int o = 16; o >= L; o >>= 1) {
            gl[e] += __shfl_xor_sync(0xffffffffu, gl[e], o);
            gh[e] += __shfl_xor_sync(0xffffffffu, gh[e], o);
        }
    if (threadIdx.x % 32 < L && lane * 16 < p.D) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            part[threadIdx.x / 32][8 * lane + e] = gl[e];
            part[threadIdx.x / 32][half + 8 * lane + e] = gh[e];
        }
    }
    __syncthreads();
    if ((int)threadIdx.x < p.D) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) s += part[w][threadIdx.x];
        p.partial[(size_t)blockIdx.x * p.D + threadIdx.x] = s;
    }
}

// dw of both tensors from the blocks' partial rows: a block takes eight features of one tensor, 32 threads a feature.
__global__ void __launch_bounds__(256) dw_kernel(const float *partial, int D, int q_blocks, int blocks, float *dw_q, float *dw_k) {
    __shared__ float part[32][9];
    const int f = threadIdx.x % 8, i = threadIdx.x / 8, col = blockIdx.x * 8 + f;
    const int b0 = blockIdx.y ? q_blocks : 0, b1 = blockIdx.y ? blocks : q_blocks;
    float s = 0.f;
#pragma unroll 8
    for (int b = b0 + i; b < b1; b += 32) s += partial[(size_t)b * D + col];
    part[i][f] = s;
    __syncthreads();
    if (i == 0) {
        for (int k = 1; k < 32; ++k) s += part[k][f];
        (blockIdx.y ? dw_k : dw_q)[col] = s;
    }
}

int lanes_of(int D) {
    int l = 1;
    while (l * 16 < D) l *= 2;
    return l;
}

constexpr int kBwdBlocks = 148 * 2;                // one wave at two blocks per SM

// What both directions share: supported sizes, the geometry and the split into work items.
int fill(const basp_plan *p, const void *w_q, const void *w_k, const float *cos, const float *sin, float eps, int want_blocks,
         NormRopeParams *prm) {
    if (p->D % 16 != 0 || p->D > 128) return BASP_ERR_UNSUPPORTED;
    if (!(eps > 0.f) || !(eps <= 3.0e38f)) return BASP_ERR_INVALID;
    if ((long long)p->Bl * p->T >= (1ll << 30)) return BASP_ERR_UNSUPPORTED;
    prm->cos = cos; prm->sin = sin; prm->eps = eps; prm->inv_D = 1.0f / (float)p->D;
    prm->D = p->D; prm->S = p->S; prm->T = p->T; prm->T_last = p->T_last; prm->K = p->K; prm->Bl = p->Bl; prm->N = p->N;
    prm->div_T = make_fastdiv((uint32_t)p->T); prm->div_T_last = make_fastdiv((uint32_t)p->T_last);
    prm->t[0].w = (const __nv_bfloat16 *)w_q; prm->t[0].heads = p->Hq;
    prm->t[1].w = (const __nv_bfloat16 *)w_k; prm->t[1].heads = p->Hkv;
    const int tokens = kThreads / lanes_of(p->D);
    prm->tiles = (p->Bl * p->T + tokens - 1) / tokens;
    // Few tokens: a token's heads are spread over blocks until the grid is want_blocks; many: one block takes them all
    const long long units = (long long)p->N * prm->tiles;
    const int heads = p->Hq + p->Hkv;
    long long per = units * heads / want_blocks;
    per = per < 1 ? 1 : (per > heads ? heads : per);
    prm->chunk_heads = (int)per;
    long long items = 0;
    for (HeadSet &t : prm->t) {
        t.chunks = (t.heads + prm->chunk_heads - 1) / prm->chunk_heads;
        items += units * t.chunks;
        if (&t == &prm->t[0]) prm->q_items = (int)items;
    }
    if (items >= (1ll << 31)) return BASP_ERR_UNSUPPORTED;
    prm->items = (int)items;
    return BASP_OK;
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

template <typename F>
int by_lanes(int D, F &&f) {
    switch (lanes_of(D)) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 4: return f(std::integral_constant<int, 4>{});
        default: return f(std::integral_constant<int, 8>{});
    }
}

}  // namespace

extern "C" int basp_qk_norm_rope(const basp_plan *p, const void *const *q_seq, const void *const *k_seq, const void *w_q,
                                 const void *w_k, const float *rope_cos, const float *rope_sin, float eps, void *const *q_out,
                                 void *const *k_out, void *stream) {
    if (!p) return BASP_ERR_NULL;
    NormRopeParams prm;
    BASP_TRY(fill(p, w_q, w_k, rope_cos, rope_sin, eps, 148 * 16, &prm));
    SpanSet spans;
    BASP_TRY(add_tables(p, &spans, w_q, w_k, rope_cos, rope_sin));
    BASP_TRY(add_shards(p, &spans, p->Hq, q_seq, false, 0, prm.t[0].x));
    BASP_TRY(add_shards(p, &spans, p->Hkv, k_seq, false, 1, prm.t[1].x));
    BASP_TRY(add_shards(p, &spans, p->Hq, q_out, true, 0, const_cast<const __nv_bfloat16 **>(prm.t[0].out)));
    BASP_TRY(add_shards(p, &spans, p->Hkv, k_out, true, 1, const_cast<const __nv_bfloat16 **>(prm.t[1].out)));
    BASP_TRY(spans.overlaps());
    return by_lanes(p->D, [&](auto lanes) -> int {
        norm_rope_kernel<decltype(lanes)::value><<<prm.items, kThreads, 0, (cudaStream_t)stream>>>(prm);
        BASP_CUDA_TRY(cudaGetLastError());
        basp_count_launch(1);
        return BASP_OK;
    });
}

extern "C" size_t basp_qk_norm_rope_bwd_workspace_bytes(const basp_plan *p) {
    return p ? (size_t)(kBwdBlocks + 1) * p->D * 4 : 0;
}

extern "C" int basp_qk_norm_rope_bwd(const basp_plan *p, const void *const *q_seq, const void *const *k_seq, const void *w_q,
                                     const void *w_k, const float *rope_cos, const float *rope_sin, float eps,
                                     const void *const *dq_out, const void *const *dk_out, void *const *dq_seq,
                                     void *const *dk_seq, float *dw_q, float *dw_k, void *workspace, size_t workspace_bytes,
                                     void *stream) {
    if (!p) return BASP_ERR_NULL;
    NormRopeParams prm;
    BASP_TRY(fill(p, w_q, w_k, rope_cos, rope_sin, eps, kBwdBlocks * 4, &prm));
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
    BASP_TRY(spans.add_out(workspace, basp_qk_norm_rope_bwd_workspace_bytes(p)));
    if (workspace_bytes < basp_qk_norm_rope_bwd_workspace_bytes(p)) return BASP_ERR_WORKSPACE;
    BASP_TRY(spans.overlaps());
    // blocks in proportion to the tensors' vectors, at least one each
    const int total = prm.items < kBwdBlocks ? prm.items : kBwdBlocks;
    int q_blocks = (int)((long long)total * p->Hq / (p->Hq + p->Hkv));
    q_blocks = q_blocks < 1 ? 1 : (q_blocks > prm.q_items ? prm.q_items : q_blocks);
    int k_blocks = total - q_blocks;
    k_blocks = k_blocks < 1 ? 1 : (k_blocks > prm.items - prm.q_items ? prm.items - prm.q_items : k_blocks);
    prm.q_blocks = q_blocks;
    prm.partial = (float *)workspace;
    const int blocks = q_blocks + k_blocks;
    return by_lanes(p->D, [&](auto lanes) -> int {
        norm_rope_bwd_kernel<decltype(lanes)::value><<<blocks, kThreads, 0, (cudaStream_t)stream>>>(prm);
        BASP_CUDA_TRY(cudaGetLastError());
        dw_kernel<<<dim3(p->D / 8, 2), 256, 0, (cudaStream_t)stream>>>(prm.partial, p->D, q_blocks, blocks, dw_q, dw_k);
        BASP_CUDA_TRY(cudaGetLastError());
        basp_count_launch(2);
        return BASP_OK;
    });
}
