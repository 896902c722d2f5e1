// The edge between two blocks on all ranks' sequence shards, one pass over the rows (`hidden` features each):
//
//   z = y w_post r_y,  h = x + s g z,  n = h w_pre r_h          r_t = (mean t^2 + eps)^(-1/2)
//   backward:  dh = dh_out + r_h dn w_pre - h r_h^3 (dn w_pre . h) / hidden = dx,   dw_pre += dn h r_h
//              dg += s dh z,   dz = s g dh,   dw_post += dz y r_y,   dy = r_y dz w_post - y r_y^3 (dz w_post . y) / hidden
//
// HBM-bound: 4 bytes read and 4 written per feature forward, 8 read and 4 written backward.  A row is contiguous, so it comes by bulk
// copies of whole rows into a ring in shared memory, asked for ahead by one thread: no registers wait for memory, and the sums
// between (two rounds over the block for each row) run under the copies.  A thread keeps its features of the row as packed bf16 and,
// backward, the three weight sums of its features in registers over all of its rows; at the end a block writes one partial row, and a
// second launch adds those in a fixed order (the same inputs give the same bits).
// A group of warps works on a row: one warp up to 512 features (eight rows at a time in a block), a whole block above.
// 64K rows of 4096, calls back to back: forward 372 us (5.8 TB/s), backward 600 us (5.4 TB/s; 836 before its sums were packed and its
// shuffles shared).
#include <cuda_bf16.h>

#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"
#include "spans.h"

int *basp_status_device_ptr();

namespace {

using namespace ptx;

constexpr int kMaxHidden = 16384;
constexpr int kMaxStages = 4;
constexpr int kMaxWarps = 16;
constexpr int kWarpRows = 8;               // groups of a block where a warp holds a row
constexpr int kMaxSmem = 225 * 1024;       // of a block, beside its barriers and sums
constexpr int kRingBytes = 192 * 1024;     // of all blocks of an SM, weights included

// R: room for ranks (8 or BASP_MAX_RANKS; a launch takes longer the larger its parameters)
template <int R>
struct NormParams {
    const __nv_bfloat16 *in[4][R];         // forward: x, y; backward: h, y, dh_out, dn
    __nv_bfloat16 *out[2][R];              // forward: h, n; backward: dx, dy
    const __nv_bfloat16 *w[3];             // w_post, gate, w_pre (nullptr: not there)
    float *partial;                        // backward: [blocks][3][hidden]; nullptr without weights
    int has[4];                            // which of the inputs are read
    int n_in;                              // how many
    float scale, eps, inv;                 // inv: 1 / hidden
    int hidden, K, stages;
    uint32_t rows_full, rows_last, rows;   // of a rank, of a group's last rank, of all (full ones)
    FastDiv div_rows, div_K;
    int *status;
};

__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
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
__device__ __forceinline__ uint64_t both(float v) { return pack_f2(v, v); }
__device__ __forceinline__ F8 ones() { return F8{{both(1.f), both(1.f), both(1.f), both(1.f)}}; }
__device__ __forceinline__ float sum2(uint64_t v) {
    float lo, hi;
    unpack_f2(v, lo, hi);
    return lo + hi;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// What a block keeps in shared memory besides the ring and the weights.
struct NormShared {
    uint64_t full[kWarpRows][kMaxStages];
    __nv_bfloat16 *to[kWarpRows][kMaxStages][2];  // where the row of a stage goes; nullptr: there is no such row
    alignas(16) float red[4][3][kMaxWarps];       // sums of the warps, in turn
    int abort_flag;
};

// Everyone of the group is here; returns whether one of them is `broken`.
template <bool kWarp>
__device__ __forceinline__ bool group_sync(bool broken) {
    if constexpr (kWarp) return __any_sync(0xffffffffu, broken);
    else return __syncthreads_or(broken);
}
// Sums over the warp of three values per thread, the k-th one in the lanes with lane % 4 == k: two steps halve what a lane carries, three
// more go over the lanes that carry the same.
__device__ __forceinline__ float warp_sum3(float a, float b, float c) {
    const int lane = threadIdx.x & 31;
    const bool odd = lane & 1, upper = lane & 2;
    // lanes with bit 0 keep b (and nothing), the others a and c
    const float keep = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
    const float other = (odd ? 0.f : c) + __shfl_xor_sync(0xffffffffu, odd ? c : 0.f, 1);
    float v = (upper ? other : keep) + __shfl_xor_sync(0xffffffffu, upper ? keep : other, 2);
#pragma unroll
    for (int o = 4; o <= 16; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sums over the group of n (1 or 3) values per thread, in all of its threads.  kWarp: the group is a warp.
template <bool kWarp, int n>
__device__ __forceinline__ bool group_sum(float (&v)[n], float (*red)[kMaxWarps], bool broken = false) {
    float mine;
    if constexpr (n == 3) mine = warp_sum3(v[0], v[1], v[2]);
    else mine = warp_sum(v[0]);
    if constexpr (kWarp) {
        if constexpr (n == 3)
#pragma unroll
            for (int i = 0; i < n; ++i) v[i] = __shfl_sync(0xffffffffu, mine, i);
        else v[0] = mine;
        __syncwarp();
        return group_sync<true>(broken);
    } else {
        const int warp = threadIdx.x / 32, warps = blockDim.x / 32, lane = threadIdx.x % 32;
        if (lane < n) red[lane][warp] = mine;
        broken = group_sync<false>(broken);
        // (the places of warps that are not there hold zeros)
        uint64_t s[n];
#pragma unroll
        for (int i = 0; i < n; ++i) s[i] = 0;
        for (int k = 0; k < warps; k += 4)
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const ulonglong2 f = *reinterpret_cast<const ulonglong2 *>(&red[i][k]);
                s[i] = add2(s[i], add2(f.x, f.y));
            }
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = sum2(s[i]);
        return broken;
    }
}

// Where the row `i` of all ranks' (full) rows lies: rank and row there, false where the rank has no such row.
template <int R>
__device__ __forceinline__ bool place_of(const NormParams<R> &p, uint32_t i, uint32_t &r, size_t &off) {
    r = fdiv(i, p.div_rows);
    const uint32_t row = i - r * p.rows_full, g = fdiv(r, p.div_K);
    off = (size_t)row * p.hidden;
    return row < ((int)(r - g * p.K) == p.K - 1 ? p.rows_last : p.rows_full);
}

// kBwd: which pass; kWarp: a warp holds a row; V: vectors of eight features per thread
template <bool kBwd, bool kWarp, int V, int R>
__global__ void __launch_bounds__(kWarp ? 32 * kWarpRows : 512, kWarp || (!kBwd && V < 4) ? 2 : 1) block_norm_kernel(const __grid_constant__ NormParams<R> p) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ NormShared sh;
    const int warp = threadIdx.x / 32, group = kWarp ? warp : 0, groups = kWarp ? kWarpRows : 1;
    const int lanes = kWarp ? 32 : (int)blockDim.x, lane = kWarp ? (int)threadIdx.x % 32 : (int)threadIdx.x;
    const uint32_t row_bytes = (uint32_t)p.hidden * 2;
    uint8_t *weights = smem, *ring = smem + 3 * row_bytes + (size_t)group * p.stages * p.n_in * row_bytes;
    for (int i = threadIdx.x; i < 4 * 3 * kMaxWarps; i += blockDim.x) (&sh.red[0][0][0])[i] = 0.f;
    if (threadIdx.x == 0) {
        sh.abort_flag = 0;
        for (int g = 0; g < groups; ++g)
            for (int s = 0; s < p.stages; ++s) mbar_init(&sh.full[g][s], 1);
        fence_mbar_init();
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (p.w[k])
            for (int i = threadIdx.x; i < p.hidden / 8; i += blockDim.x)
                reinterpret_cast<uint4 *>(weights + k * row_bytes)[i] = __ldg(reinterpret_cast<const uint4 *>(p.w[k]) + i);
    if (kBwd) allow_next_kernel();
    __syncthreads();
    const uint32_t step = gridDim.x * groups, first = blockIdx.x * groups + group;
    // One thread of the group asks for the rows, a ring ahead.  `i`: the row, s: its stage
    auto ask = [&](uint32_t i, int s) {
        uint32_t r;
        size_t off;
        if (i >= p.rows) return;
        const bool there = place_of(p, i, r, off);
        // (forward without a block before: no sum is written, and the place only says that the row is there)
        sh.to[group][s][0] = there ? (p.out[0][r] ? p.out[0][r] : p.out[1][r]) + off : nullptr;
        sh.to[group][s][1] = there && p.out[1][r] ? p.out[1][r] + off : nullptr;
        if (!there) {                              // a short last rank: nothing comes
            mbar_arrive(&sh.full[group][s]);
            return;
        }
        mbar_arrive_expect_tx(&sh.full[group][s], p.n_in * row_bytes);
        uint8_t *to = ring + (size_t)s * p.n_in * row_bytes;
#pragma unroll
        for (int k = 0; k < (kBwd ? 4 : 2); ++k)
            if (p.has[k]) {
                bulk_load(to, p.in[k][r] + off, row_bytes, &sh.full[group][s]);
                to += row_bytes;
            }
    };
    if (lane == 0)
        for (int s = 0; s < p.stages; ++s) ask(first + s * step, s);

    const bool post = p.w[0], gated = p.w[1], pre = p.w[2];
    uint64_t acc[kBwd ? 3 : 1][kBwd ? V : 1][4];     // pairs of the three weight sums
    if constexpr (kBwd)
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[k][v][e] = 0;
    const auto weight = [&](int k, int v) { return widen(reinterpret_cast<const uint4 *>(weights + k * row_bytes)[lane + v * lanes]); };
    const uint64_t scale2 = both(p.scale);

    int stage = 0;
    uint32_t phases = 0, turn = 0;                 // a bit for each stage
    bool broken = false;
    for (uint32_t i = first; i < p.rows; i += step, ++turn) {
        const int at = stage;
        stage = stage + 1 == p.stages ? 0 : stage + 1;
        if (!mbar_wait(&sh.full[group][at], (phases >> at) & 1, &sh.abort_flag)) {
            if (atomicCAS(p.status, 0, 6) == 0) { p.status[1] = 1; p.status[2] = (int)blockIdx.x; p.status[3] = (int)i; }
            sh.abort_flag = 1;
            broken = true;                         // the group leaves together, at its next meeting and before it stores anything
        }
        __nv_bfloat16 *const out0 = sh.to[group][at][0], *const out1 = sh.to[group][at][1];
        phases ^= 1u << at;
        uint4 raw[kBwd ? 4 : 2][V];
        {
            const uint8_t *from = ring + (size_t)at * p.n_in * row_bytes;
#pragma unroll
            for (int k = 0; k < (kBwd ? 4 : 2); ++k) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    raw[k][v] = make_uint4(0, 0, 0, 0);
                    if (p.has[k] && (lane + v * lanes) * 8 < p.hidden) raw[k][v] = reinterpret_cast<const uint4 *>(from)[lane + v * lanes];
                }
                if (p.has[k]) from += row_bytes;
            }
        }
        float (*red)[3][kMaxWarps] = sh.red + 2 * (turn & 1);
        if constexpr (!kBwd) {
            float ry = 1.f, sums[1];
            if (post) {
                uint64_t sq = 0;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const F8 y = widen(raw[1][v]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sq = fma2(y.p[e], y.p[e], sq);
                }
                sums[0] = sum2(sq);
                broken = group_sum<kWarp>(sums, red[0], broken);
                ry = rsqrtf(fmaf(sums[0], p.inv, p.eps));
            } else {
                if constexpr (kWarp) __syncwarp();
                broken = group_sync<kWarp>(broken);
            }
            if (broken) break;
            if (lane == 0) ask(i + p.stages * step, at);       // everyone has its part of the row
            if (!out0) continue;
            const uint64_t ry2 = both(ry);
            uint64_t sq = 0;
            F8 h[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                h[v] = widen(raw[0][v]);
                const bool mine = (lane + v * lanes) * 8 < p.hidden;
                if (p.has[1] && mine) {
                    const F8 y = widen(raw[1][v]), wp = post ? weight(0, v) : ones(), g = gated ? weight(1, v) : ones();
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[v].p[e] = fma2(mul2(g.p[e], scale2), mul2(mul2(y.p[e], ry2), wp.p[e]), h[v].p[e]);
                    st16(out0 + (lane + v * lanes) * 8, narrow(h[v]));
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) sq = fma2(h[v].p[e], h[v].p[e], sq);
            }
            if (pre) {
                sums[0] = sum2(sq);
                group_sum<kWarp>(sums, red[1]);
                const uint64_t rh2 = both(rsqrtf(fmaf(sums[0], p.inv, p.eps)));
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if ((lane + v * lanes) * 8 < p.hidden) {
                        const F8 w = weight(2, v);
                        F8 n;
#pragma unroll
                        for (int e = 0; e < 4; ++e) n.p[e] = mul2(mul2(h[v].p[e], rh2), w.p[e]);
                        st16(out1 + (lane + v * lanes) * 8, narrow(n));
                    }
            }
        } else {
            // sums of y^2, h^2 and dn w_pre h
            uint64_t s0 = 0, s1 = 0, s2 = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if ((lane + v * lanes) * 8 >= p.hidden) continue;
                const F8 y = widen(raw[1][v]);
#pragma unroll
                for (int e = 0; e < 4; ++e) s0 = fma2(y.p[e], y.p[e], s0);
                if (pre) {
                    const F8 h = widen(raw[0][v]), dn = widen(raw[3][v]), w = weight(2, v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s1 = fma2(h.p[e], h.p[e], s1);
                        s2 = fma2(mul2(dn.p[e], w.p[e]), h.p[e], s2);
                    }
                }
            }
            float sums[3] = {sum2(s0), sum2(s1), sum2(s2)};
            broken = group_sum<kWarp>(sums, red[0], broken);
            if (broken) break;
            if (lane == 0) ask(i + p.stages * step, at);       // everyone has its part of the row
            if (!out0) continue;
            const float ry = post ? rsqrtf(fmaf(sums[0], p.inv, p.eps)) : 1.f, rh = rsqrtf(fmaf(sums[1], p.inv, p.eps));
            // in this order: r^3 alone leaves fp32 for zeros and a tiny eps
            const uint64_t rh2 = both(rh), ch2 = both(-(rh * sums[2] * p.inv) * rh * rh), ry2 = both(ry);
            F8 dz[V];
            uint64_t s3 = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if ((lane + v * lanes) * 8 >= p.hidden) continue;
                F8 dh = widen(raw[2][v]);
                if (pre) {
                    const F8 h = widen(raw[0][v]), dn = widen(raw[3][v]), w = weight(2, v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t t = mul2(dn.p[e], rh2);
                        acc[2][v][e] = fma2(t, h.p[e], acc[2][v][e]);
                        dh.p[e] = add2(dh.p[e], fma2(t, w.p[e], mul2(h.p[e], ch2)));
                    }
                }
                st16(out0 + (lane + v * lanes) * 8, narrow(dh));
                if (!out1) continue;
                const F8 y = widen(raw[1][v]), wp = post ? weight(0, v) : ones(), g = gated ? weight(1, v) : ones();
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t u = mul2(dh.p[e], scale2), yr = mul2(y.p[e], ry2);
                    acc[1][v][e] = fma2(u, mul2(yr, wp.p[e]), acc[1][v][e]);
                    const uint64_t d = mul2(u, g.p[e]);
                    acc[0][v][e] = fma2(d, yr, acc[0][v][e]);
                    dz[v].p[e] = mul2(d, wp.p[e]);
                    s3 = fma2(dz[v].p[e], y.p[e], s3);
                }
                if (!post) st16(out1 + (lane + v * lanes) * 8, narrow(dz[v]));
            }
            if (post) {
                float dot[1] = {sum2(s3)};
                group_sum<kWarp>(dot, red[1]);
                const uint64_t cy2 = both(-(ry * dot[0] * p.inv) * ry * ry);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if ((lane + v * lanes) * 8 < p.hidden) {
                        const F8 y = widen(raw[1][v]);
                        F8 dy;
#pragma unroll
                        for (int e = 0; e < 4; ++e) dy.p[e] = fma2(dz[v].p[e], ry2, mul2(y.p[e], cy2));
                        st16(out1 + (lane + v * lanes) * 8, narrow(dy));
                    }
            }
        }
    }
    if (sh.abort_flag) {                           // let copies that are still in flight land before the shared memory is given back
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) { }
    }
    if constexpr (kBwd) {
        if (!p.partial) return;                    // no weights, no sums
        float *to = p.partial + (size_t)blockIdx.x * 3 * p.hidden;
        if constexpr (kWarp) {                     // the groups' sums added one after another where the weights were
            float *sum = reinterpret_cast<float *>(smem);        // [3][hidden]: 3 rows of 4 bytes where 3 of 2 and a ring were
            for (int g = 0; g < groups; ++g) {
                __syncthreads();
                if (g == group)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if ((lane + v * lanes) * 8 < p.hidden)
#pragma unroll
                            for (int k = 0; k < 3; ++k)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    uint64_t *f = reinterpret_cast<uint64_t *>(sum + k * p.hidden + (lane + v * lanes) * 8 + 2 * e);
                                    *f = g == 0 ? acc[k][v][e] : add2(*f, acc[k][v][e]);
                                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < 3 * p.hidden; i += blockDim.x) to[i] = sum[i];
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if ((lane + v * lanes) * 8 < p.hidden)
#pragma unroll
                    for (int k = 0; k < 3; ++k) {
                        ulonglong2 *f = reinterpret_cast<ulonglong2 *>(to + (size_t)k * p.hidden + (lane + v * lanes) * 8);
                        f[0] = make_ulonglong2(acc[k][v][0], acc[k][v][1]);
                        f[1] = make_ulonglong2(acc[k][v][2], acc[k][v][3]);
                    }
        }
    }
}

// The weights' gradients from the blocks' partial rows: a block takes eight features of one of them, 32 threads a feature.
__global__ void __launch_bounds__(256) norm_dw_kernel(const float *partial, int hidden, int blocks, float *dw_post, float *dgate, float *dw_pre) {
    __shared__ float part[32][9];
    float *to = blockIdx.y == 0 ? dw_post : blockIdx.y == 1 ? dgate : dw_pre;
    wait_previous_kernel();
    if (!to) return;
    const int f = threadIdx.x % 8, i = threadIdx.x / 8, col = blockIdx.x * 8 + f;
    float s = 0.f;
#pragma unroll 8
    for (int b = i; b < blocks; b += 32) s += partial[((size_t)b * 3 + blockIdx.y) * hidden + col];
    part[i][f] = s;
    __syncthreads();
    if (i == 0) {
        for (int k = 1; k < 32; ++k) s += part[k][f];
        to[col] = s;
    }
}

struct NormShape {
    int vectors, threads, stages, wave;            // per thread, per block, of the ring, blocks of a full GPU
    size_t smem;
};
// One warp a row up to 512 features, one vector a lane up to 256.  Above that a block: what a row costs beside its features (its place, its
// sums over the block) is paid by every warp, so two vectors a thread (four above 8192 features: 512 threads), but forward, where
// a block of two warps would be the measure, one up to 2048 (64K rows of 1024 / 2048 / 4096 forward: one vector 100 / 191 / 395 us,
// two 112 / 202 / 372).  Blocks per SM by the registers, 128 and 64 a thread.
NormShape shape_of(int hidden, int n_in, bool bwd) {
    NormShape s;
    const int nv = hidden / 8;
    const bool warp = nv <= 64;
    s.vectors = warp ? (nv <= 32 ? 1 : 2) : !bwd && nv <= 256 ? 1 : nv <= 1024 ? 2 : 4;
    s.threads = warp ? 32 * kWarpRows : 32 * ((nv + 32 * s.vectors - 1) / (32 * s.vectors));
    const int resident = bwd || s.vectors == 4 ? 512 : !warp ? 1024 : s.vectors == 1 ? 1024 : 768;      // threads of an SM
    int per_sm = resident / s.threads;
    if (per_sm < 1) per_sm = 1;
    const size_t row = (size_t)hidden * 2, stage = row * (n_in < 1 ? 1 : n_in) * (warp ? kWarpRows : 1);
    while (per_sm > 1 && kRingBytes / per_sm < (long long)(3 * row + 2 * stage)) --per_sm;
    long long stages = ((long long)kRingBytes / per_sm - (long long)(3 * row)) / (long long)stage;
    s.stages = stages < 1 ? 1 : stages > kMaxStages ? kMaxStages : (int)stages;
    s.wave = 148 * per_sm;
    s.smem = 3 * row + s.stages * stage;
    if (bwd && warp && s.smem < 3 * row * 2) s.smem = 3 * row * 2;      // the groups' fp32 sums
    return s;
}

int supported(int hidden, float eps, float scale) {
    if (hidden <= 0) return BASP_ERR_INVALID;
    if (hidden % 8 != 0 || hidden > kMaxHidden) return BASP_ERR_UNSUPPORTED;
    if (!(eps > 0.f && eps <= 3.0e38f) || !(scale >= -3.0e38f && scale <= 3.0e38f)) return BASP_ERR_INVALID;
    return BASP_OK;
}

template <bool kBwd, int R>
int launch(const basp_plan *pl, NormParams<R> &prm, int hidden, cudaStream_t st, int *blocks) {
    prm.status = basp_status_device_ptr();
    if (!prm.status) return BASP_ERR_CUDA;
    prm.hidden = hidden; prm.inv = 1.0f / (float)hidden; prm.K = pl->K;
    prm.n_in = 0;
    for (int k = 0; k < 4; ++k) prm.n_in += prm.has[k];
    const long long rows = (long long)pl->Bl * pl->T;
    if (rows * pl->N >= (1ll << 31) - (1 << 20)) return BASP_ERR_UNSUPPORTED;
    prm.rows_full = (uint32_t)rows; prm.rows_last = (uint32_t)((long long)pl->Bl * pl->T_last); prm.rows = (uint32_t)(rows * pl->N);
    prm.div_rows = make_fastdiv(prm.rows_full); prm.div_K = make_fastdiv((uint32_t)pl->K);
    const NormShape s = shape_of(hidden, prm.n_in, kBwd);
    prm.stages = s.stages;
    const bool warp = s.threads == 32 * kWarpRows && hidden <= 512;
    const long long units = warp ? (prm.rows + kWarpRows - 1) / kWarpRows : prm.rows;
    *blocks = (int)(units < s.wave ? units : s.wave);
    const auto go = [&](auto vectors, auto warp_tag) -> int {
        constexpr auto kernel = block_norm_kernel<kBwd, decltype(warp_tag)::value, decltype(vectors)::value, R>;
        BASP_TRY((allow_smem<block_norm_kernel<kBwd, decltype(warp_tag)::value, decltype(vectors)::value, R>, kMaxSmem>()));
        kernel<<<*blocks, s.threads, s.smem, st>>>(prm);
        BASP_CUDA_TRY(cudaGetLastError());
        basp_count_launch(1);
        return BASP_OK;
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if (warp) return s.vectors == 1 ? go(One{}, std::true_type{}) : go(Two{}, std::true_type{});
    if constexpr (!kBwd)
        if (s.vectors == 1) return go(One{}, std::false_type{});
    return s.vectors == 2 ? go(Two{}, std::false_type{}) : go(Four{}, std::false_type{});
}

// Adds one tensor's shards to the spans and the parameter block
int add_shards(const basp_plan *p, SpanSet *s, int hidden, const void *const *shards, bool out, int slot, const __nv_bfloat16 **to) {
    if (!shards) return BASP_ERR_NULL;
    for (int r = 0; r < p->N; ++r) {
        const size_t bytes = (size_t)p->Bl * basp_rank_tokens(p, r % p->K) * hidden * 2;
        BASP_TRY(out ? s->add_out(shards[r], bytes, 16, slot * BASP_MAX_RANKS + r) : s->add_in(shards[r], bytes, 16, slot * BASP_MAX_RANKS + r));
        to[r] = (const __nv_bfloat16 *)shards[r];
    }
    return BASP_OK;
}

template <int R>
int run_fwd(const basp_plan *p, int hidden, const void *const *x_seq, const void *const *y_seq, const void *w_post, const void *gate,
            const void *w_pre, float res_scale, float eps, void *const *h_seq, void *const *n_seq, cudaStream_t st) {
    NormParams<R> prm{};
    SpanSet spans;
    const void *w[3] = {w_post, gate, w_pre};
    for (int k = 0; k < 3; ++k)
        if (w[k]) {
            BASP_TRY(spans.add_in(w[k], (size_t)hidden * 2));
            prm.w[k] = (const __nv_bfloat16 *)w[k];
        }
    BASP_TRY(add_shards(p, &spans, hidden, x_seq, false, 0, prm.in[0]));
    if (y_seq) BASP_TRY(add_shards(p, &spans, hidden, y_seq, false, 0, prm.in[1]));
    // a row is read whole before any of it is written: an output may be either input
    if (h_seq) BASP_TRY(add_shards(p, &spans, hidden, h_seq, true, 0, const_cast<const __nv_bfloat16 **>(prm.out[0])));
    if (n_seq) BASP_TRY(add_shards(p, &spans, hidden, n_seq, true, 0, const_cast<const __nv_bfloat16 **>(prm.out[1])));
    BASP_TRY(spans.overlaps());
    prm.has[0] = 1; prm.has[1] = y_seq != nullptr;
    prm.scale = res_scale; prm.eps = eps;
    int blocks;
    return launch<false, R>(p, prm, hidden, st, &blocks);
}

// A partial row of three sums for each block (the fewest inputs leave room for the most blocks).
size_t bwd_workspace_bytes(int hidden) { return (size_t)shape_of(hidden, 0, true).wave * 3 * hidden * 4; }

template <int R>
int run_bwd(const basp_plan *p, int hidden, const void *const *h_seq, const void *const *y_seq, const void *w_post, const void *gate,
            const void *w_pre, float res_scale, float eps, const void *const *dh_out, const void *const *dn, void *const *dx_seq,
            void *const *dy_seq, float *dw_post, float *dgate, float *dw_pre, void *workspace, size_t workspace_bytes, cudaStream_t st) {
    NormParams<R> prm{};
    SpanSet spans;
    const void *w[3] = {w_post, gate, w_pre};
    float *dw[3] = {dw_post, dgate, dw_pre};
    for (int k = 0; k < 3; ++k)
        if (w[k]) {
            BASP_TRY(spans.add_in(w[k], (size_t)hidden * 2));
            prm.w[k] = (const __nv_bfloat16 *)w[k];
            if (dw[k]) BASP_TRY(spans.add_out(dw[k], (size_t)hidden * 4, 4));
        }
    if (w_pre) BASP_TRY(add_shards(p, &spans, hidden, h_seq, false, 3, prm.in[0]));
    if (w_post || gate) BASP_TRY(add_shards(p, &spans, hidden, y_seq, false, 1, prm.in[1]));
    if (dh_out) BASP_TRY(add_shards(p, &spans, hidden, dh_out, false, 0, prm.in[2]));
    if (w_pre) BASP_TRY(add_shards(p, &spans, hidden, dn, false, 0, prm.in[3]));
    BASP_TRY(add_shards(p, &spans, hidden, dx_seq, true, 0, const_cast<const __nv_bfloat16 **>(prm.out[0])));
    if (dy_seq) BASP_TRY(add_shards(p, &spans, hidden, dy_seq, true, 1, const_cast<const __nv_bfloat16 **>(prm.out[1])));
    const bool weights = w_post || gate || w_pre;
    if (weights) {
        BASP_TRY(spans.add_out(workspace, bwd_workspace_bytes(hidden)));
        if (workspace_bytes < bwd_workspace_bytes(hidden)) return BASP_ERR_WORKSPACE;
    }
    BASP_TRY(spans.overlaps());
    prm.has[0] = prm.has[3] = w_pre != nullptr;
    prm.has[1] = w_post || gate;
    prm.has[2] = dh_out != nullptr;
    prm.partial = weights ? (float *)workspace : nullptr;       // (without weights nothing is known of the workspace)
    prm.scale = res_scale; prm.eps = eps;
    int blocks;
    BASP_TRY((launch<true, R>(p, prm, hidden, st, &blocks)));
    if (weights) {
        BASP_CUDA_TRY(launch_early(norm_dw_kernel, dim3(hidden / 8, 3), 256, st, (const float *)prm.partial, hidden, blocks,
                                   w_post ? dw_post : (float *)nullptr, gate ? dgate : (float *)nullptr, w_pre ? dw_pre : (float *)nullptr));
        basp_count_launch(1);
    }
    return BASP_OK;
}

}  // namespace

extern "C" int basp_block_norm(const basp_plan *p, int hidden, const void *const *x_seq, const void *const *y_seq, const void *w_post,
                               const void *gate, const void *w_pre, float res_scale, float eps, void *const *h_seq,
                               void *const *n_seq, void *stream) {
    if (!p || !x_seq) return BASP_ERR_NULL;
    // what goes together: the sum h with y, its norm and gate with y, n with its weight; and there has to be something to do
    if ((y_seq != nullptr) != (h_seq != nullptr) || (w_pre != nullptr) != (n_seq != nullptr)) return BASP_ERR_NULL;
    if (!y_seq && (w_post || gate || !w_pre)) return BASP_ERR_NULL;
    BASP_TRY(supported(hidden, eps, res_scale));
    return p->N <= 8 ? run_fwd<8>(p, hidden, x_seq, y_seq, w_post, gate, w_pre, res_scale, eps, h_seq, n_seq, (cudaStream_t)stream)
                     : run_fwd<BASP_MAX_RANKS>(p, hidden, x_seq, y_seq, w_post, gate, w_pre, res_scale, eps, h_seq, n_seq,
                                               (cudaStream_t)stream);
}

extern "C" size_t basp_block_norm_bwd_workspace_bytes(const basp_plan *p, int hidden) {
    return p && supported(hidden, 1.f, 1.f) == BASP_OK ? bwd_workspace_bytes(hidden) : 0;
}

extern "C" int basp_block_norm_bwd(const basp_plan *p, int hidden, const void *const *h_seq, const void *const *y_seq, const void *w_post,
                                   const void *gate, const void *w_pre, float res_scale, float eps, const void *const *dh_out,
                                   const void *const *dn, void *const *dx_seq, void *const *dy_seq, float *dw_post, float *dgate,
                                   float *dw_pre, void *workspace, size_t workspace_bytes, void *stream) {
    if (!p || !dx_seq || (!dh_out && !w_pre)) return BASP_ERR_NULL;
    // every weight with its gradient; the gradients of the block's output and of its norm and gate come together
    if ((w_post != nullptr) != (dw_post != nullptr) || (gate != nullptr) != (dgate != nullptr) || (w_pre != nullptr) != (dw_pre != nullptr))
        return BASP_ERR_NULL;
    if ((w_pre != nullptr) != (dn != nullptr) || (!dy_seq && (w_post || gate))) return BASP_ERR_NULL;
    BASP_TRY(supported(hidden, eps, res_scale));
    return p->N <= 8 ? run_bwd<8>(p, hidden, h_seq, y_seq, w_post, gate, w_pre, res_scale, eps, dh_out, dn, dx_seq, dy_seq, dw_post,
                                  dgate, dw_pre, workspace, workspace_bytes, (cudaStream_t)stream)
                     : run_bwd<BASP_MAX_RANKS>(p, hidden, h_seq, y_seq, w_post, gate, w_pre, res_scale, eps, dh_out, dn, dx_seq, dy_seq,
                                               dw_post, dgate, dw_pre, workspace, workspace_bytes, (cudaStream_t)stream);
}
