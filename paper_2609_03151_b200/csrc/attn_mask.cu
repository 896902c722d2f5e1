// The mask object: per-query key ranges to the tables that the masked attention kernels walk (attn_mask.cuh).
//
//   basp_mask_ranges   the ranges as they are given
//   basp_mask_packed   from the positions inside packed documents:  begin = max(i - pos, i - window + 1),
//                      end = max(i + 1, i - pos + prefix),  nothing where pos < 0
//
// Three steps, each over warps: a warp takes a query tile (its rows' ranges and their extremes), then a key tile (which query
// tiles see it), then a work item (its place in the order, longest first, by counting the longer ones: the place does not depend
// on timing).  Up to 64 tiles one block does all three, above that they are three launches that start early.  The tables are a
// few kilobytes: what bounds the calls is latency (two sequences of 777 tokens: 14 tiles in
// one launch, 4.3 us; in three launches 8.6).
#include <type_traits>

#include "attn_mask.cuh"
#include "common.cuh"
#include "ptx.cuh"
#include "spans.h"

namespace {

using namespace ptx;

constexpr int kSmallTiles = 64;     // one block of 32 warps, up to two tiles each
constexpr int kBigWarps = 8;

struct MaskParams {
    const int *begin, *end;                    // basp_mask_ranges
    const int *positions, *prefix;             // basp_mask_packed (prefix may be nullptr)
    int2 *range;
    MaskTile *tiles;
    int2 *seen;
    MaskFwdEntry *fwd;
    MaskBwdEntry *bwd;
    int B, S, n_tiles, n_blocks, window;
};

__device__ __forceinline__ int clamp_to(long long v, int hi) { return (int)(v < 0 ? 0 : v > hi ? hi : v); }

// Ranges of the rows of a query tile and their extremes.
__device__ __forceinline__ MaskTile tile_step(const MaskParams &p, int idx, int lane) {
    const int seq = idx / p.n_tiles, tile = idx - seq * p.n_tiles;
    int lo_min = p.S, lo_max = 0, hi_min = p.S, hi_max = 0;
    // the loads of all four rows first (positions and prefix, or begin and end)
    const int *one = p.positions ? p.positions : p.begin, *other = p.positions ? p.prefix : p.end;
    int u[kMaskTile / 32], v[kMaskTile / 32];
#pragma unroll
    for (int k = 0; k < kMaskTile / 32; ++k) {
        const int i = tile * kMaskTile + k * 32 + lane;
        const size_t at = (size_t)seq * p.S + i;
        u[k] = i < p.S ? one[at] : -1;
        v[k] = i < p.S && other ? other[at] : 0;
    }
#pragma unroll
    for (int k = 0; k < kMaskTile / 32; ++k) {
        const int i = tile * kMaskTile + k * 32 + lane;
        int lo = 0, hi = 0;
        if (i < p.S) {
            if (p.positions) {
                const int pos = u[k];
                if (pos >= 0) {
                    long long first = (long long)i - pos, past = (long long)i + 1;
                    if (p.prefix) past = max(past, first + v[k]);
                    if (p.window > 0) first = max(first, (long long)i - p.window + 1);
                    lo = clamp_to(first, p.S);
                    hi = clamp_to(past, p.S);
                }
            } else {
                lo = clamp_to(u[k], p.S);
                hi = clamp_to(v[k], p.S);
            }
            if (hi <= lo) lo = hi = 0;
            if (hi > lo) { lo_min = min(lo_min, lo); hi_max = max(hi_max, hi); }
            lo_max = max(lo_max, lo);
            hi_min = min(hi_min, hi);
        }
        p.range[((size_t)seq * p.n_tiles + tile) * kMaskTile + k * 32 + lane] = make_int2(lo, hi);
    }
    lo_min = __reduce_min_sync(0xffffffffu, lo_min);
    lo_max = __reduce_max_sync(0xffffffffu, lo_max);
    hi_min = __reduce_min_sync(0xffffffffu, hi_min);
    hi_max = __reduce_max_sync(0xffffffffu, hi_max);
    MaskTile t{0, 0, 0, 0};
    if (hi_max > lo_min) {
        t.begin = lo_min / kMaskTile;
        t.end = (hi_max + kMaskTile - 1) / kMaskTile;
        t.full = (lo_max + kMaskTile - 1) / kMaskTile;
        t.full_end = hi_min / kMaskTile;
    }
    if (lane == 0) p.tiles[idx] = t;
    return t;
}

// The query tiles that see a key tile.  `tiles`, here and below, and `seen`: p's own, or copies in shared memory.
__device__ __forceinline__ int2 seen_step(const MaskParams &p, const MaskTile *tiles, int idx, int lane) {
    const int seq = idx / p.n_tiles, n = idx - seq * p.n_tiles;
    int first = p.n_tiles, last = 0;
    for (int m = lane; m < p.n_tiles; m += 32) {
        const MaskTile t = tiles[seq * p.n_tiles + m];
        if (t.begin <= n && n < t.end) { first = min(first, m); last = m + 1; }
    }
    first = __reduce_min_sync(0xffffffffu, first);
    last = __reduce_max_sync(0xffffffffu, last);
    const int2 range = last > 0 ? make_int2(first, last) : make_int2(0, 0);
    if (lane == 0) p.seen[idx] = range;
    return range;
}

// The place of a work item of either pass among all of its pass.
template <typename F>
__device__ __forceinline__ int place_of(int mine, int count, int lane, F &&cost_of) {
    const int cost = cost_of(mine);
    int before = 0;
    for (int e = lane; e < count; e += 32) {
        const int c = cost_of(e);
        before += c > cost || (c == cost && e < mine);
    }
    return __reduce_add_sync(0xffffffffu, before);
}
__device__ __forceinline__ int fwd_cost(const MaskParams &p, const MaskTile *tiles, int e) {
    const int seq = e / p.n_blocks, tile = 2 * (e - seq * p.n_blocks);
    const MaskTile a = tiles[seq * p.n_tiles + tile];
    const MaskTile b = tile + 1 < p.n_tiles ? tiles[seq * p.n_tiles + tile + 1] : MaskTile{0, 0, 0, 0};
    return a.end - a.begin + b.end - b.begin;
}
__device__ __forceinline__ void order_step(const MaskParams &p, const MaskTile *tiles, const int2 *seen, int idx, int lane) {
    const int n_fwd = p.B * p.n_blocks, n_bwd = p.B * p.n_tiles;
    if (idx < n_fwd) {
        const int place = place_of(idx, n_fwd, lane, [&](int e) { return fwd_cost(p, tiles, e); });
        if (lane == 0) {
            MaskFwdEntry e{};
            e.seq = idx / p.n_blocks;
            e.block = idx - e.seq * p.n_blocks;
            const int tile = e.seq * p.n_tiles + 2 * e.block;
            e.tile[0] = tiles[tile];
            if (2 * e.block + 1 < p.n_tiles) e.tile[1] = tiles[tile + 1];
            p.fwd[place] = e;
        }
    } else {
        const int i = idx - n_fwd, place = place_of(i, n_bwd, lane, [&](int e) { return seen[e].y - seen[e].x; });
        if (lane == 0) {
            const int2 s = seen[i];
            p.bwd[place] = MaskBwdEntry{i / p.n_tiles, i % p.n_tiles, s.x, s.y};
        }
    }
}

__global__ void __launch_bounds__(1024) mask_small_kernel(const __grid_constant__ MaskParams p) {
    __shared__ MaskTile tiles[kSmallTiles];
    __shared__ int2 seen[kSmallTiles];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
    const int n = p.B * p.n_tiles, items = n + p.B * p.n_blocks;
    allow_next_kernel();
    for (int i = warp; i < n; i += warps) {
        const MaskTile t = tile_step(p, i, lane);
        if (lane == 0) tiles[i] = t;
    }
    __syncthreads();
    for (int i = warp; i < n; i += warps) {
        const int2 s = seen_step(p, tiles, i, lane);
        if (lane == 0) seen[i] = s;
    }
    __syncthreads();
    for (int i = warp; i < items; i += warps) order_step(p, tiles, seen, i, lane);
}

template <int kStep>
__global__ void __launch_bounds__(32 * kBigWarps) mask_step_kernel(const __grid_constant__ MaskParams p, int items) {
    const int idx = blockIdx.x * kBigWarps + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (kStep > 0) wait_previous_kernel();
    allow_next_kernel();
    if (idx >= items) return;
    if (kStep == 0) tile_step(p, idx, lane);
    if (kStep == 1) seen_step(p, p.tiles, idx, lane);
    if (kStep == 2) order_step(p, p.tiles, p.seen, idx, lane);
}

int mask_launch(const basp_plan *pl, MaskParams &p, void *mask, cudaStream_t st) {
    const MaskLayout l = mask_layout(pl);
    char *m = (char *)mask;
    p.range = (int2 *)m;
    p.tiles = (MaskTile *)(m + l.tiles);
    p.seen = (int2 *)(m + l.seen);
    p.fwd = (MaskFwdEntry *)(m + l.fwd);
    p.bwd = (MaskBwdEntry *)(m + l.bwd);
    p.B = pl->B; p.S = pl->S; p.n_tiles = l.n_tiles; p.n_blocks = l.n_blocks;
    const long long n = (long long)pl->B * l.n_tiles, items = n + (long long)pl->B * l.n_blocks;
    if (items >= (1ll << 30)) return BASP_ERR_UNSUPPORTED;
    if (n <= kSmallTiles) {
        mask_small_kernel<<<1, 32 * (int)(items < 32 ? items : 32), 0, st>>>(p);
        BASP_CUDA_TRY(cudaGetLastError());
        basp_count_launch(1);
        return BASP_OK;
    }
    const auto blocks = [](long long warps) { return dim3((unsigned)((warps + kBigWarps - 1) / kBigWarps)); };
    mask_step_kernel<0><<<blocks(n), 32 * kBigWarps, 0, st>>>(p, (int)n);
    BASP_CUDA_TRY(cudaGetLastError());
    BASP_CUDA_TRY(launch_early(mask_step_kernel<1>, blocks(n), 32 * kBigWarps, st, p, (int)n));
    BASP_CUDA_TRY(launch_early(mask_step_kernel<2>, blocks(items), 32 * kBigWarps, st, p, (int)items));
    basp_count_launch(3);
    return BASP_OK;
}

}  // namespace

int basp_score_args(const basp_plan *p, const basp_score *score, float scale, ScoreArgs *out) {
    *out = ScoreArgs{};
    out->B = p->B;
    if (!score) return BASP_ERR_NULL;
    if (!(score->softcap >= 0.f && score->softcap <= 3.0e38f)) return BASP_ERR_INVALID;
    if (score->softcap > 0.f) {
        const double in = (double)scale / score->softcap, log2e = 1.4426950408889634;
        // (the kernels take one and the other, and its square and that's reciprocal, as fp32 numbers)
        if (!(in >= 1e-9 && in <= 1e6 && score->softcap >= 1e-12f && score->softcap <= 1e12f)) return BASP_ERR_INVALID;
        out->cap_in = (float)in;
        out->cap_out = (float)(score->softcap * log2e);
        const double c[5] = {0.999999846, -0.333315002, 0.132978737, -0.0515179165, 0.0146250855};
        double power = scale * log2e;                       // softcap log2(e) in^(2k + 1)
        for (int k = 0; k < 5; ++k, power *= in * in) out->near[k] = (float)(c[k] * power);
        // the coefficients have to be normal fp32 numbers: where the last one is not, it and the one before are not needed up to 0.05; for
        // in above 1e3 they overflow
        out->near_limit = in > 1e3 ? -1.f : (float)((out->near[4] < 1.2e-38f ? 0.05 : 0.65) / in);
    }
    if ((uintptr_t)score->slopes & 3) return BASP_ERR_ALIGN;
    out->slopes = score->slopes;
    if (score->mask) {
        const MaskLayout l = mask_layout(p);
        if ((uintptr_t)score->mask & 15) return BASP_ERR_ALIGN;
        if (score->mask_bytes < l.bytes) return BASP_ERR_WORKSPACE;
        const char *m = (const char *)score->mask;
        out->range = (const int2 *)m;
        out->tiles = (const MaskTile *)(m + l.tiles);
        out->fwd = (const MaskFwdEntry *)(m + l.fwd);
        out->bwd = (const MaskBwdEntry *)(m + l.bwd);
    }
    return BASP_OK;
}

extern "C" size_t basp_mask_bytes(const basp_plan *p) { return p ? mask_layout(p).bytes : 0; }

extern "C" int basp_mask_ranges(const basp_plan *p, const int *key_begin, const int *key_end, void *mask, size_t mask_bytes,
                                void *stream) {
    if (!p) return BASP_ERR_NULL;
    SpanSet spans;
    BASP_TRY(spans.add_in(key_begin, (size_t)p->B * p->S * 4, 4));
    BASP_TRY(spans.add_in(key_end, (size_t)p->B * p->S * 4, 4));
    BASP_TRY(spans.add_out(mask, basp_mask_bytes(p)));
    if (mask_bytes < basp_mask_bytes(p)) return BASP_ERR_WORKSPACE;
    BASP_TRY(spans.overlaps());
    MaskParams prm{};
    prm.begin = key_begin;
    prm.end = key_end;
    return mask_launch(p, prm, mask, (cudaStream_t)stream);
}

extern "C" int basp_mask_packed(const basp_plan *p, const int *positions, const int *prefix, int window, void *mask,
                                size_t mask_bytes, void *stream) {
    if (!p) return BASP_ERR_NULL;
    if (window < 0 || !p->causal) return BASP_ERR_INVALID;
    SpanSet spans;
    BASP_TRY(spans.add_in(positions, (size_t)p->B * p->S * 4, 4));
    if (prefix) BASP_TRY(spans.add_in(prefix, (size_t)p->B * p->S * 4, 4));
    BASP_TRY(spans.add_out(mask, basp_mask_bytes(p)));
    if (mask_bytes < basp_mask_bytes(p)) return BASP_ERR_WORKSPACE;
    BASP_TRY(spans.overlaps());
    MaskParams prm{};
    prm.positions = positions;
    prm.prefix = prefix;
    prm.window = window;
    return mask_launch(p, prm, mask, (cudaStream_t)stream);
}
