// The mask object of the masked attention: what basp_mask_ranges and basp_mask_packed write into the caller's buffer and the
// attention kernels read.  A query i of sequence b sees the keys [begin, end) of its range; everything else here follows from
// the ranges and says which 128 x 128 tiles there are anything to do in.
#pragma once
#include <cuda_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "plan.h"

constexpr int kMaskTile = 128;

// Key tiles of a query tile: [begin, end) hold every key that one of its rows sees, in [full, full_end) every row sees every key.
struct MaskTile { int begin, end, full, full_end; };
// 256 query rows (two tiles) of a sequence as a work item of the forward pass.
struct MaskFwdEntry { int seq, block, pad[2]; MaskTile tile[2]; };
// A key tile of a sequence as a work item of the backward pass: the query tiles [first, last) see some of it.
struct MaskBwdEntry { int seq, tile, first, last; };

struct MaskLayout {
    int n_tiles, n_blocks;                             // of one sequence
    size_t tiles, seen, fwd, bwd, bytes;               // offsets behind the ranges, which start the buffer
};

// ranges int2 [B][n_tiles * 128] | MaskTile [B][n_tiles] | int2 [B][n_tiles] (query tiles that see a key tile) |
// MaskFwdEntry [B * n_blocks], longest first | MaskBwdEntry [B * n_tiles], longest first
inline MaskLayout mask_layout(const basp_plan *p) {
    MaskLayout l;
    l.n_tiles = (p->S + kMaskTile - 1) / kMaskTile;
    l.n_blocks = (l.n_tiles + 1) / 2;
    const size_t t = (size_t)p->B * l.n_tiles;
    l.tiles = t * kMaskTile * 8;
    l.seen = l.tiles + t * sizeof(MaskTile);
    l.fwd = (l.seen + t * 8 + 15) & ~(size_t)15;
    l.bwd = l.fwd + (size_t)p->B * l.n_blocks * sizeof(MaskFwdEntry);
    l.bytes = l.bwd + t * sizeof(MaskBwdEntry);
    return l;
}

// How the kernels of both directions see a call's basp_score.
struct ScoreArgs {
    const int2 *range;              // nullptr: no mask object, the plan's own mask
    const MaskTile *tiles;
    const MaskFwdEntry *fwd;
    const MaskBwdEntry *bwd;
    const float *slopes;            // [Hq]
    float cap_in, cap_out;          // scale / softcap and softcap * log2(e); 0: no cap
    float near[5], near_limit;      // coefficients of the capped score near zero (score.cuh), and up to which raw score
    int B;
};

// f(kCap, kBias) with the two as compile-time truth values
template <typename F>
int dispatch_score(bool cap, bool bias, F &&f) {
    if (cap) return bias ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
    return bias ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

inline float resolved_scale(const basp_plan *p, float softmax_scale) { return softmax_scale == 0.f ? 1.f / sqrtf((float)p->D) : softmax_scale; }

// Checks a basp_score and fills in what the kernels take of it (attn_mask.cu).
int basp_score_args(const basp_plan *p, const basp_score *score, float scale, ScoreArgs *out);

// What basp_attn_masked_fwd and _bwd refuse, found without a launch (the layer asks before its first exchange).
int basp_attn_masked_fwd_check(const basp_plan *pl, const basp_score *score, const void *const *q_head, const void *const *k_head,
                               const void *const *v_head, void *const *o_head, float *const *lse_shards, float softmax_scale);
int basp_attn_masked_bwd_check(const basp_plan *pl, const basp_score *score, const void *const *q_head, const void *const *k_head,
                               const void *const *v_head, const void *const *o_head, const void *const *do_head,
                               const float *const *lse_shards, void *const *dq_head, void *const *dk_head, void *const *dv_head,
                               void *workspace, size_t workspace_bytes, float softmax_scale);
