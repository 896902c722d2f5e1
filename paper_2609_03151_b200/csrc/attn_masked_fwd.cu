// Attention with masked and shaped scores over each virtual rank's head slice, forward:
//
//   z_ij = c tanh(scale q_i.k_j / c) - slope_h |i - j|   (c = 0: no cap),   visible: begin_i <= j < end_i
//   O_i = sum_j softmax_j(z_ij) v_j,  LSE_i = ln sum_j exp(z_ij);  a row that sees no key: O = 0, LSE = -inf
//
// The structure is that of the causal kernel (attn_fwd_ws.cuh: one persistent CTA of 512 threads per SM, two 128-row query
// tiles on one stream of K/V tiles, softmax / correction / TMA / two MMA warps, one score buffer, P in TMEM, every wait
// bounded).  What is different:
//   - a query tile has key tiles [begin, end) of its own, read from the mask object; the two tiles of an item may have
//     different ones, or none.  Tiles outside are neither loaded nor multiplied, so the work follows the documents.
//   - only tiles that are not wholly visible are masked, with the bounds of the thread's row.  A row can meet such a
//     tile before it has seen any key: its reference stays -inf and its exponentials are taken against 0.
//   - items are dealt longest first in the mask object's order.
// Scores, maxima, sums and O are fp32; P becomes bf16 as an operand of the second product (the tensor cores take no wider one at their full
// rate) while its sum is that of the unrounded exponentials, and O is rounded once at the end.  O is off by 0.0019 to 0.0024 (2-norm), where the
// exact result rounded to bf16 is by 0.0017.
// Capped or biased scores have a kernel of their own (attn_shaped_fwd.cuh): four softmax warpgroups instead of two.  For plain scores two
// are better (16K causal tokens, 32/8 heads of 128: 1.55-1.7 ms and 1.8; through a mask object 1.72).
#include <cuda.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"
#include "tmap.cuh"
#include "attn_common.cuh"
#include "attn_mask.cuh"
#include "score.cuh"
#include "spans.h"

int *basp_status_device_ptr();

namespace {

constexpr int kMfThreads = 512;
constexpr int kMfStages = 4;             // K/V ring slots (one 128 x D tile each)
constexpr float kMfRescale = 8.f;        // how far (log2) a row's maximum may pass its reference before O is rescaled

template <int R>
struct MaskedFwdParams {
    CUtensorMap q[R], k[R], v[R];
    __nv_bfloat16 *o[R];
    float *lse[R];
    ScoreArgs score;
    int K, Bl, S, Hq, Hq_l, Hkv_l, n_tiles, n_blocks, total;   // total: work items
    int Dg;                      // head dimension in memory; the tile loads zero-fill the columns past it
    int causal, has_lse;         // causal: of the plan, where there is no mask object
    float scale_log2;            // softmax scale * log2(e)
    int *status;
    FastDiv div_items, div_hq_l, div_q_per_kv, div_B, div_bl;
};

struct MfItem {
    int r, bl, seq, h, hkv, block;
    MaskTile t[2];
    int j0, j1;                  // key tiles of the item: those of its query tiles and what lies between
};

template <int R>
__device__ __forceinline__ MaskTile mf_plain_tile(const MaskedFwdParams<R> &p, int tile) {
    MaskTile t{0, 0, 0, 0};
    if (tile < p.n_tiles) {
        t.end = p.causal ? tile + 1 : p.n_tiles;
        t.full_end = p.causal ? tile : p.S / kTile;
    }
    return t;
}
__device__ __forceinline__ void mf_clamp(MaskTile &t, int n_tiles) {       // whatever the buffer holds, no tile outside the tensors
    t.begin = max(t.begin, 0);
    t.end = min(t.end, n_tiles);
}

template <int R>
__device__ __forceinline__ bool mf_get_item(const MaskedFwdParams<R> &p, int round, MfItem &it) {
    const int pos = (round & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x;   // boustrophedon
    const int i = round * (int)gridDim.x + pos;
    if (i >= p.total) return false;
    // the heads of a block of query rows side by side: neighbouring CTAs read the same K/V tiles through L2
    const int e = (int)fdiv((uint32_t)i, p.div_items);
    const int head = i - e * p.Hq, l = (int)fdiv((uint32_t)head, p.div_hq_l);
    it.h = head - l * p.Hq_l;
    it.hkv = (int)fdiv((uint32_t)it.h, p.div_q_per_kv);
    if (p.score.range) {
        const MaskFwdEntry *at = p.score.fwd + e;
        const int4 *from = reinterpret_cast<const int4 *>(at);
        const int4 a = ld_written(from), b = ld_written(from + 1), c = ld_written(from + 2);
        it.seq = min(max(a.x, 0), p.score.B - 1);
        it.block = min(max(a.y, 0), p.n_blocks - 1);
        it.t[0] = MaskTile{b.x, b.y, b.z, b.w};
        it.t[1] = MaskTile{c.x, c.y, c.z, c.w};
        mf_clamp(it.t[0], p.n_tiles);
        mf_clamp(it.t[1], p.n_tiles);
    } else {
        const int back = (int)fdiv((uint32_t)e, p.div_B);
        it.seq = e - back * p.score.B;
        it.block = p.n_blocks - 1 - back;
        it.t[0] = mf_plain_tile(p, 2 * it.block);
        it.t[1] = mf_plain_tile(p, 2 * it.block + 1);
    }
    const int g = (int)fdiv((uint32_t)it.seq, p.div_bl);
    it.bl = it.seq - g * p.Bl;
    it.r = g * p.K + l;
    const bool a0 = it.t[0].begin < it.t[0].end, a1 = it.t[1].begin < it.t[1].end;
    it.j0 = a0 ? (a1 ? min(it.t[0].begin, it.t[1].begin) : it.t[0].begin) : it.t[1].begin;
    it.j1 = a0 ? (a1 ? max(it.t[0].end, it.t[1].end) : it.t[0].end) : it.t[1].end;
    return true;
}

struct MfShared {
    uint64_t q_full, q_empty;
    uint64_t kv_full[kMfStages], kv_empty[kMfStages];
    uint64_t s_free, pv_done[2];
    uint64_t alpha_full[2][2];       // [tile][step parity]
    uint64_t s_full[2], p_full[2], o_rescaled[2], o_final[2], o_free[2];
    uint64_t l_full[2][2];           // [tile][item parity]
    float alpha[2][2][kTile];        // [tile][step parity][row]
    float l[2][2][kTile];            // [item parity][tile][row]
    uint32_t tmem_base;
    int abort_flag;
};

constexpr uint32_t kMfSleepNs = 32;      // back-off of the correction and producer warps while they wait

#define MF_WAIT(bar, parity, role, detail)                                     \
    do {                                                                        \
        if (!mbar_wait((bar), (parity), &sh.abort_flag, ((role) >= 20 && (role) < 40) ? kMfSleepNs : 0)) { \
            sh.abort_flag = 1;                                                  \
            report(p.status, 5, (role), (detail));                              \
            goto mf_done;                                                       \
        }                                                                       \
    } while (0)

template <int D, int R>
__global__ void __launch_bounds__(kMfThreads, 1) attn_masked_fwd_kernel(const __grid_constant__ MaskedFwdParams<R> p) {
    constexpr int kSlabs = D / 64;
    constexpr int kTileBytes = kTile * D * 2;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sQ = smem;                                // 2 tiles
    uint8_t *sKV = smem + 2 * kTileBytes;              // kMfStages tiles
    __shared__ MfShared sh;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

    if (tid == 0) {
        mbar_init(&sh.q_full, 1);
        mbar_init(&sh.q_empty, 1);
        for (int i = 0; i < kMfStages; ++i) { mbar_init(&sh.kv_full[i], 1); mbar_init(&sh.kv_empty[i], 1); }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&sh.s_full[t], 1);
            mbar_init(&sh.alpha_full[t][0], 4);
            mbar_init(&sh.alpha_full[t][1], 4);
            mbar_init(&sh.p_full[t], 4);
            mbar_init(&sh.o_rescaled[t], 4);
            mbar_init(&sh.o_final[t], 1);
            mbar_init(&sh.l_full[t][0], 4);
            mbar_init(&sh.l_full[t][1], 4);
            mbar_init(&sh.o_free[t], 4);
        }
        mbar_init(&sh.s_free, 4);
        mbar_init(&sh.pv_done[0], 1);
        mbar_init(&sh.pv_done[1], 1);
        sh.abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 12) { tmem_alloc(&sh.tmem_base, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    wait_previous_kernel();        // (nothing of another kernel's was touched up to here)
    allow_next_kernel();
    // One score tile S at columns 0..127 (the two query tiles take turns), P_t at 128 + 64 t, O_t at 256 + 128 t.

    if (warp < 8) {
        // =============================================================== softmax of query tile t
        reg_inc<192>();
        const int t = warp >> 2;
        const int row = tid & 127;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t S_a = tmem + lane_addr;                   // the shared score tile
        const uint32_t P_t = tmem + 128 + 64 * t + lane_addr;
        uint32_t it_cnt = 0, ep_cnt = 0;
        MfItem item;
        for (int round = 0; mf_get_item(p, round, item); ++round) {
            const int qt = 2 * item.block + t, begin = t ? item.t[1].begin : item.t[0].begin, end = t ? item.t[1].end : item.t[0].end;
            const int full = t ? item.t[1].full : item.t[0].full, full_end = t ? item.t[1].full_end : item.t[0].full_end;
            if (qt >= p.n_tiles) continue;
            const int s_pos = qt * kTile + row;
            float *lse_at = p.has_lse && s_pos < p.S ? p.lse[item.r] + ((size_t)item.bl * p.Hq_l + item.h) * p.S + s_pos : nullptr;
            if (begin >= end) {                                  // no row of the tile sees a key
                if (lse_at) *lse_at = -INFINITY;
                continue;
            }
            // keys [lo, hi) of this thread's row
            int lo = 0, hi = 0;
            if (p.score.range) {
                const int2 range = ld_written(p.score.range + ((size_t)item.seq * p.n_tiles + qt) * kTile + row);
                lo = range.x;
                hi = range.y;
            } else if (s_pos < p.S) {
                hi = p.causal ? s_pos + 1 : p.S;
            }
            float m_ref = -INFINITY, l_run = 0.f;
            for (int j = begin; j < end; ++j, ++it_cnt) {
                MF_WAIT(&sh.s_full[t], it_cnt & 1, 10 + t, j);
                tc_fence_after();
                uint32_t s[kTile];
                tmem_ld_x32(S_a + 0, *reinterpret_cast<uint32_t(*)[32]>(&s[0]));
                tmem_ld_x32(S_a + 32, *reinterpret_cast<uint32_t(*)[32]>(&s[32]));
                tmem_ld_x32(S_a + 64, *reinterpret_cast<uint32_t(*)[32]>(&s[64]));
                tmem_ld_x32(S_a + 96, *reinterpret_cast<uint32_t(*)[32]>(&s[96]));
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.s_free);       // the scores are in registers: the other tile's Q.K^T may overwrite S
                if (__builtin_expect(j < full || j >= full_end, 0)) {     // keys outside of [lo, hi) are hidden
                    const int first = lo - j * kTile, past = hi - j * kTile;
                    if (__any_sync(0xffffffffu, first > 0)) {
#pragma unroll
                        for (int i = 0; i < kTile; ++i)
                            if (i < first) s[i] = 0xff800000u;   // -inf
                    }
                    if (__any_sync(0xffffffffu, past < kTile)) {
#pragma unroll
                        for (int i = 0; i < kTile; ++i)
                            if (i >= past) s[i] = 0xff800000u;
                    }
                }
                float mxs[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) mxs[i] = max3(__uint_as_float(s[i]), __uint_as_float(s[8 + i]), __uint_as_float(s[16 + i]));
#pragma unroll
                for (int i = 24; i + 15 < kTile; i += 16)
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        mxs[k] = max3(mxs[k], __uint_as_float(s[i + k]), __uint_as_float(s[i + 8 + k]));
#pragma unroll
                for (int k = 0; k < 8; ++k) mxs[k] = fmaxf(mxs[k], __uint_as_float(s[120 + k]));
                const float mx = fmaxf(fmaxf(fmaxf(mxs[0], mxs[1]), fmaxf(mxs[2], mxs[3])),
                                       fmaxf(fmaxf(mxs[4], mxs[5]), fmaxf(mxs[6], mxs[7]))) * p.scale_log2;
                float alpha = 1.f;
                if (mx > m_ref + kMfRescale) { alpha = exp2_approx(m_ref - mx); m_ref = mx; }
                sh.alpha[t][it_cnt & 1][row] = alpha;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.alpha_full[t][it_cnt & 1]);
                const float m_sub = m_ref == -INFINITY ? 0.f : m_ref;      // no key yet: every exponential is exp2(-inf) = 0
                uint64_t rs2[2] = {0ull, 0ull};
                const uint64_t sc2 = both(p.scale_log2), nm2 = both(-m_sub);
#pragma unroll
                for (int i = 0; i < kTile; i += 2) {
                    float x0, x1;
                    unpack_f2(fma2(pack_f2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), sc2, nm2), x0, x1);
                    const float e0 = exp2_approx(x0), e1 = exp2_approx(x1);
                    rs2[(i >> 1) & 1] = add2(rs2[(i >> 1) & 1], pack_f2(e0, e1));
                    s[i >> 1] = pack_bf16x2(e0, e1);
                }
                // the previous P_t V has read P_t before this step's replaces it
                if (it_cnt > 0) { MF_WAIT(&sh.pv_done[t], (it_cnt - 1) & 1, 14 + t, j); tc_fence_after(); }
                tmem_st_x32(P_t + 0, *reinterpret_cast<const uint32_t(*)[32]>(&s[0]));
                tmem_st_x32(P_t + 32, *reinterpret_cast<const uint32_t(*)[32]>(&s[32]));
                float ra, rb;
                unpack_f2(add2(rs2[0], rs2[1]), ra, rb);
                l_run = l_run * alpha + (ra + rb);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_full[t]);
            }
            // one key: P is a rounded number that the sum below it has to be too, so that O is the key's value
            sh.l[ep_cnt & 1][t][row] = hi - lo == 1 ? round_bf16(l_run) : l_run;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.l_full[t][ep_cnt & 1]);
            ++ep_cnt;
            if (lse_at) *lse_at = l_run == 0.f ? -INFINITY : m_ref * 0.6931471805599453f + logf(l_run);
        }
    } else if (warp < 12) {
        // =============================================================== correction + epilogue
        reg_dec<64>();
        const int row = tid & 127;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        uint32_t it_cnt[2] = {0, 0}, ep_cnt[2] = {0, 0};
        MfItem item;
        for (int round = 0; mf_get_item(p, round, item); ++round) {
            for (int j = item.j0; j < item.j1; ++j) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (j < item.t[t].begin || j >= item.t[t].end) continue;
                    MF_WAIT(&sh.alpha_full[t][it_cnt[t] & 1], (it_cnt[t] >> 1) & 1, 20 + t, j);
                    const float alpha = sh.alpha[t][it_cnt[t] & 1][row];
                    ++it_cnt[t];
                    // O_t is only ours once P_t V(j-1) has completed
                    const bool begun = j > item.t[t].begin;
                    if (begun) MF_WAIT(&sh.pv_done[t], (it_cnt[t] - 2) & 1, 22 + t, j);
                    if (begun && !__all_sync(0xffffffffu, alpha == 1.f)) {
                        tc_fence_after();
                        const uint32_t O_t = tmem + 256 + 128 * t + lane_addr;
#pragma unroll 1                 // rare and not time-critical: kept small
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t rr[32];
                            tmem_ld_x32(O_t + c * 32, rr);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) rr[i] = __float_as_uint(__uint_as_float(rr[i]) * alpha);
                            tmem_st_x32(O_t + c * 32, rr);
                        }
                        tmem_wait_st();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.o_rescaled[t]);
                }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int qt = 2 * item.block + t;
                if (qt >= p.n_tiles) continue;
                const bool in_seq = qt * kTile + row < p.S;                 // rows past a ragged end are not stored
                __nv_bfloat16 *dst = p.o[item.r] + (((size_t)item.bl * p.S + (size_t)qt * kTile + row) * p.Hq_l + item.h) * p.Dg;
                if (item.t[t].begin >= item.t[t].end) {
                    if (in_seq)
                        for (int c = 0; c < p.Dg; c += 8) *reinterpret_cast<uint4 *>(dst + c) = make_uint4(0, 0, 0, 0);
                    continue;
                }
                MF_WAIT(&sh.l_full[t][ep_cnt[t] & 1], (ep_cnt[t] >> 1) & 1, 24 + t, 0);
                MF_WAIT(&sh.o_final[t], ep_cnt[t] & 1, 26 + t, 0);
                const float l = sh.l[ep_cnt[t] & 1][t][row];
                const float inv_l = l == 0.f ? 0.f : 1.f / l;               // a row without a key: P was zero throughout
                ++ep_cnt[t];
                tc_fence_after();
                const uint32_t O_t = tmem + 256 + 128 * t + lane_addr;
#pragma unroll
                for (int cc = 0; cc < D / 32; ++cc) {
                    if (cc * 32 >= p.Dg) break;          // columns past the real head dimension are zero padding
                    uint32_t rr[32];
                    tmem_ld_x32(O_t + cc * 32, rr);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint4 o4;
                        o4.x = pack_bf16x2(__uint_as_float(rr[8 * i + 0]) * inv_l, __uint_as_float(rr[8 * i + 1]) * inv_l);
                        o4.y = pack_bf16x2(__uint_as_float(rr[8 * i + 2]) * inv_l, __uint_as_float(rr[8 * i + 3]) * inv_l);
                        o4.z = pack_bf16x2(__uint_as_float(rr[8 * i + 4]) * inv_l, __uint_as_float(rr[8 * i + 5]) * inv_l);
                        o4.w = pack_bf16x2(__uint_as_float(rr[8 * i + 6]) * inv_l, __uint_as_float(rr[8 * i + 7]) * inv_l);
                        if (in_seq && cc * 32 + i * 8 < p.Dg) *reinterpret_cast<uint4 *>(dst + cc * 32 + i * 8) = o4;
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.o_free[t]);
            }
        }
    } else {
        reg_dec<64>();
        if (warp == 12) {
            // =========================================================== TMA producer (lane 0 issues)
            uint32_t kv_it = 0, item_n = 0;
            MfItem item;
            for (int round = 0; mf_get_item(p, round, item); ++round) {
                if (item.j0 >= item.j1) continue;
                MF_WAIT(&sh.q_empty, (item_n & 1) ^ 1, 30, round);
                ++item_n;
                const int n_q = 2 * item.block + 1 < p.n_tiles ? 2 : 1;
                if (lane == 0) {
                    mbar_arrive_expect_tx(&sh.q_full, n_q * kTileBytes);
                    for (int t = 0; t < n_q; ++t)
                        for (int s = 0; s < kSlabs; ++s)
                            tma_load_3d(sQ + t * kTileBytes + s * 16384, &p.q[item.r], &sh.q_full, s * 64, item.h,
                                        item.bl * p.S + (2 * item.block + t) * kTile);
                }
                for (int j = item.j0; j < item.j1; ++j) {
#pragma unroll
                    for (int x = 0; x < 2; ++x, ++kv_it) {
                        const uint32_t slot = kv_it % kMfStages, ph = (kv_it / kMfStages) & 1;
                        MF_WAIT(&sh.kv_empty[slot], ph ^ 1, 31, j);
                        const CUtensorMap *tm = x == 0 ? &p.k[item.r] : &p.v[item.r];
                        if (lane == 0) {
                            mbar_arrive_expect_tx(&sh.kv_full[slot], kTileBytes);
                            for (int s = 0; s < kSlabs; ++s)
                                tma_load_3d(sKV + slot * kTileBytes + s * 16384, tm, &sh.kv_full[slot], s * 64, item.hkv,
                                            item.bl * p.S + j * kTile);
                        }
                    }
                }
            }
        } else if (warp == 13) {
            // =========================================================== MMA issuer 1: S = Q_t K_j^T (lane 0 issues)
            const uint32_t idesc_qk = make_idesc_bf16(kTile, kTile, false, false);
            uint32_t item_n = 0, qk_cnt = 0, kv_base = 0;     // K_j of the item at ring index kv_base + 2 (j - j0)
            MfItem item;
            const uint64_t desc_k = make_smem_desc_sw128(0, 16, 1024);        // K-major operands (Q, K)
            const uint32_t q_addr16 = smem_u32(sQ) >> 4, kv_addr16 = smem_u32(sKV) >> 4;
            for (int round = 0; mf_get_item(p, round, item); ++round) {
                if (item.j0 >= item.j1) continue;
                MF_WAIT(&sh.q_full, item_n & 1, 40, round);
                ++item_n;
                for (int j = item.j0; j < item.j1; ++j) {
                    const uint32_t idx = kv_base + 2 * (j - item.j0), slot = idx % kMfStages;
                    MF_WAIT(&sh.kv_full[slot], (idx / kMfStages) & 1, 41, j);
                    tc_fence_after();
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (j < item.t[t].begin || j >= item.t[t].end) continue;
                        // score tile number q may only follow the hand-over of q - 1 to its softmax warps
                        if (qk_cnt > 0) { MF_WAIT(&sh.s_free, (qk_cnt - 1) & 1, 48, j); tc_fence_after(); }
                        ++qk_cnt;
                        const uint64_t a = desc_k | (uint64_t)(q_addr16 + t * (kTileBytes >> 4));
                        const uint64_t b = desc_k | (uint64_t)(kv_addr16 + slot * (kTileBytes >> 4));
                        if (lane == 0) {
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const uint32_t off16 = ((kk / 4) * 16384 + (kk % 4) * 32) >> 4;
                                mma_ss(tmem, a + off16, b + off16, idesc_qk, kk > 0);
                            }
                            tc_commit(&sh.s_full[t]);
                        }
                    }
                    if (lane == 0) {
                        tc_commit(&sh.kv_empty[slot]);                            // K_j has no reader left
                        if (j == item.j1 - 1) tc_commit(&sh.q_empty);             // that was the item's last Q.K^T
                    }
                }
                kv_base += 2 * (item.j1 - item.j0);
            }
        } else if (warp == 14) {
            // =========================================================== MMA issuer 2: O_t += P_t V_j (lane 0 issues)
            const uint32_t idesc_pv = make_idesc_bf16(kTile, D, false, true);
            uint32_t it_cnt[2] = {0, 0}, ep_cnt[2] = {0, 0}, kv_base = 0;     // V_j at ring index kv_base + 2 (j - j0) + 1
            MfItem item;
            const uint64_t desc_v = make_smem_desc_sw128(0, 16384, 1024);     // MN-major operand (V)
            const uint32_t kv_addr16 = smem_u32(sKV) >> 4;
            for (int round = 0; mf_get_item(p, round, item); ++round) {
                if (item.j0 >= item.j1) continue;
                for (int j = item.j0; j < item.j1; ++j) {
                    const uint32_t idx = kv_base + 2 * (j - item.j0) + 1, slot = idx % kMfStages;
                    MF_WAIT(&sh.kv_full[slot], (idx / kMfStages) & 1, 42, j);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (j < item.t[t].begin || j >= item.t[t].end) continue;
                        if (j == item.t[t].begin) MF_WAIT(&sh.o_free[t], (ep_cnt[t] & 1) ^ 1, 43 + t, round);
                        MF_WAIT(&sh.p_full[t], it_cnt[t] & 1, 45 + t, j);
                        MF_WAIT(&sh.o_rescaled[t], it_cnt[t] & 1, 47 + t, j);
                        ++it_cnt[t];
                        tc_fence_after();
                        const uint64_t b = desc_v | (uint64_t)(kv_addr16 + slot * (kTileBytes >> 4));
                        if (lane == 0) {
#pragma unroll
                            for (int kk = 0; kk < kTile / 16; ++kk)
                                mma_ts(tmem + 256 + 128 * t, tmem + 128 + 64 * t + kk * 8, b + kk * (2048 >> 4), idesc_pv,
                                       (j > item.t[t].begin) || (kk > 0));
                            tc_commit(&sh.pv_done[t]);
                            if (j == item.t[t].end - 1) tc_commit(&sh.o_final[t]);
                        }
                        if (j == item.t[t].end - 1) ++ep_cnt[t];
                    }
                    if (lane == 0) tc_commit(&sh.kv_empty[slot]);                 // V_j has no reader left
                }
                kv_base += 2 * (item.j1 - item.j0);
            }
        }
    }

mf_done:
    tc_fence_before();
    __syncthreads();
    if (sh.abort_flag) {
        // let copies that are still in flight land before the shared memory is given back
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) { }
        __syncthreads();
    }
    if (warp == 12) tmem_dealloc(tmem, 512);
}

#undef MF_WAIT

#include "attn_shaped_fwd.cuh"

template <int D, int R, int kForm, bool kBias>
int sf_launch(const MaskedFwdParams<R> &prm, int grid, cudaStream_t st) {
    constexpr int smem = (2 + kMfStages) * kTile * D * 2 + 1024;
    BASP_TRY((allow_smem<attn_shaped_fwd_kernel<D, R, kForm, kBias>, smem>()));
    BASP_CUDA_TRY(launch_early_smem(attn_shaped_fwd_kernel<D, R, kForm, kBias>, dim3(grid), kSfThreads, smem, st, prm));
    basp_count_launch(1);
    return BASP_OK;
}

template <int D, int R>
int mf_launch(const MaskedFwdParams<R> &prm, int grid, cudaStream_t st) {
    constexpr int smem = (2 + kMfStages) * kTile * D * 2 + 1024;
    BASP_TRY((allow_smem<attn_masked_fwd_kernel<D, R>, smem>()));
    BASP_CUDA_TRY(launch_early_smem(attn_masked_fwd_kernel<D, R>, dim3(grid), kMfThreads, smem, st, prm));
    basp_count_launch(1);
    return BASP_OK;
}

template <int R>
int mf_run(const basp_plan *pl, const basp_score *score, const void *const *q, const void *const *k, const void *const *v,
           void *const *o, float *const *lse, float scale, cudaStream_t st) {
    MaskedFwdParams<R> prm;
    BASP_TRY(basp_score_args(pl, score, scale, &prm.score));
    const uint64_t rows = (uint64_t)pl->Bl * pl->S;
    for (int r = 0; r < pl->N; ++r) {
        BASP_TRY(tmap::encode_rows_heads_d(&prm.q[r], q[r], rows, pl->Hq_l, pl->D, kTile));
        BASP_TRY(tmap::encode_rows_heads_d(&prm.k[r], k[r], rows, pl->Hkv_l, pl->D, kTile));
        BASP_TRY(tmap::encode_rows_heads_d(&prm.v[r], v[r], rows, pl->Hkv_l, pl->D, kTile));
        prm.o[r] = (__nv_bfloat16 *)o[r];
        prm.lse[r] = lse ? lse[r] : nullptr;
    }
    prm.K = pl->K; prm.Bl = pl->Bl; prm.S = pl->S; prm.Hq = pl->Hq; prm.Hq_l = pl->Hq_l; prm.Hkv_l = pl->Hkv_l;
    prm.n_tiles = (pl->S + kTile - 1) / kTile;
    prm.n_blocks = (prm.n_tiles + 1) / 2;
    const long long total = (long long)pl->B * prm.n_blocks * pl->Hq;
    if (total >= (1ll << 31) - 4096 || rows >= (1ull << 31)) return BASP_ERR_UNSUPPORTED;      // 31-bit items and tile coordinates
    prm.total = (int)total;
    prm.Dg = pl->D;
    prm.causal = pl->causal; prm.has_lse = lse != nullptr;
    prm.scale_log2 = fmaxf(scale * 1.4426950408889634f, 1e-30f);      // (0 times a hidden score would be NaN)
    prm.status = basp_status_device_ptr();
    if (!prm.status) return BASP_ERR_CUDA;
    prm.div_items = make_fastdiv((uint32_t)pl->Hq);
    prm.div_hq_l = make_fastdiv((uint32_t)pl->Hq_l);
    prm.div_q_per_kv = make_fastdiv((uint32_t)(pl->Hq_l / pl->Hkv_l));
    prm.div_B = make_fastdiv((uint32_t)pl->B);
    prm.div_bl = make_fastdiv((uint32_t)pl->Bl);
    int sms = 0;
    BASP_TRY(sm_count(&sms));
    const int grid = (int)(total < sms ? total : sms);
    return dispatch_score(prm.score.cap_out > 0.f, prm.score.slopes != nullptr, [&](auto cap, auto bias) {
        constexpr bool kCap = decltype(cap)::value, kBias = decltype(bias)::value;
        const auto shaped = [&](auto form) {
            constexpr int kForm = decltype(form)::value;
            return pl->D > 64 ? sf_launch<128, R, kForm, kBias>(prm, grid, st) : sf_launch<64, R, kForm, kBias>(prm, grid, st);
        };
        if constexpr (kCap)
            return prm.score.cap_out <= 80.f ? shaped(std::integral_constant<int, 0>{}) : shaped(std::integral_constant<int, 2>{});
        else if constexpr (kBias)
            return shaped(std::integral_constant<int, 1>{});
        else
            return pl->D > 64 ? mf_launch<128, R>(prm, grid, st) : mf_launch<64, R>(prm, grid, st);
    });
}

}  // namespace

int basp_attn_masked_fwd_check(const basp_plan *pl, const basp_score *score, const void *const *q_head, const void *const *k_head,
                               const void *const *v_head, void *const *o_head, float *const *lse_shards, float softmax_scale) {
    if (!pl || !score || !q_head || !k_head || !v_head || !o_head) return BASP_ERR_NULL;
    if (!scale_ok(softmax_scale)) return BASP_ERR_INVALID;
    if (pl->D < 16 || pl->D > 128 || pl->D % 16 != 0) return BASP_ERR_UNSUPPORTED;
    SpanSet spans;
    const size_t rows = (size_t)pl->Bl * pl->S, q_bytes = rows * pl->Hq_l * pl->D * 2, k_bytes = rows * pl->Hkv_l * pl->D * 2;
    for (int r = 0; r < pl->N; ++r) {
        BASP_TRY(spans.add_in(q_head[r], q_bytes));
        BASP_TRY(spans.add_in(k_head[r], k_bytes));
        BASP_TRY(spans.add_in(v_head[r], k_bytes));
        BASP_TRY(spans.add_out(o_head[r], q_bytes));
        if (lse_shards) BASP_TRY(spans.add_out(lse_shards[r], rows * pl->Hq_l * 4, 4));
    }
    if (score->slopes) BASP_TRY(spans.add_in(score->slopes, (size_t)pl->Hq * 4, 4));
    if (score->mask) BASP_TRY(spans.add_in(score->mask, basp_mask_bytes(pl)));
    BASP_TRY(spans.overlaps());
    ScoreArgs args;
    return basp_score_args(pl, score, resolved_scale(pl, softmax_scale), &args);
}

extern "C" int basp_attn_masked_fwd(const basp_plan *pl, const basp_score *score, const void *const *q_head, const void *const *k_head,
                                    const void *const *v_head, void *const *o_head, float *const *lse_shards, float softmax_scale,
                                    void *stream) {
    BASP_TRY(basp_attn_masked_fwd_check(pl, score, q_head, k_head, v_head, o_head, lse_shards, softmax_scale));
    const float scale = resolved_scale(pl, softmax_scale);
    return pl->N <= 8 ? mf_run<8>(pl, score, q_head, k_head, v_head, o_head, lse_shards, scale, (cudaStream_t)stream)
                      : mf_run<BASP_MAX_RANKS>(pl, score, q_head, k_head, v_head, o_head, lse_shards, scale, (cudaStream_t)stream);
}
