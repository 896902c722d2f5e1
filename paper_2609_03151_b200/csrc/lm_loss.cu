// Softmax cross entropy of the language-model head over a large vocabulary, on all ranks' sequence shards, without keeping
// the logits; alone, and with its gradients.  For a token with hidden state x, label y and weight g:
//
//   z = x W^T,   lse = ln sum_v exp z_v,   loss = lse - z_y,
//   dz = g (softmax(z) - onehot(y)),       dx = dz W,       dW = sum_tokens dz^T x
//
// Three products, each 2 rows*vocab*hidden operations on the tensor cores, and one element-wise pass:
//   (rows)                 every row's nonzero features, see "cut off" below
//   (1) z = x W^T          epilogue: per row and 128 columns the maximum m and the sum of exp(z - m), the target's logit apart
//                          from the others; for the gradient also every logit as its distance below that maximum, 16 bits:
//                          rn((m - z) log2(e) 2^10), saturating at 2^-64 of the maximum's probability
//   (merge)                rows' statistics -> loss and lse; the target's logit summed again in fp32
//   (dz)                   in place: 16-bit distance -> bf16 dz; and the piece's rows of x side by side for (3), those without a
//                          part in the gradients as zeros (0 x NaN would reach every word's gradient)
//   (2) dx = dz W          split over the vocabulary where there are too few row tiles for all SMs (fp32 partial sums, joined by
//                          one more pass)
//   (3) dW = dz^T x        K = the piece's rows; with several pieces the sum is carried in fp32
// Tensor-bound for many rows: 8192 rows of 4096 features against 128256 words take 19.3 to 20.1 ms (1280 to 1337 TFLOP/s, at the power
// limit; the three products alone by cuBLAS 18.6 ms), of which dz takes 0.62 (4.2 GB, HBM-bound).  Several pieces: 1260 TFLOP/s, for
// the fp32 sum of dW.  Few rows: bound by reading W twice and writing dW (48 rows against 32000 words: 161 us on the GPU).  Rows are
// worked on in pieces (default 8192), so what lies between the products is 2 bytes per logit of one piece.
//
// Roundings.  A distance is off by at most 2^-11 in log2, so a probability by 2^-11 ln 2 = 3.4e-4, before it is rounded to bf16
// (2^-8) as an operand: 16 bits do for what would otherwise be an fp32 logit, twice the memory and traffic.  The target is left out of
// the sums: with o = ln sum_{v != y} exp z_v, loss = softplus(o - z_y) and the target's dz = -g sigmoid(o - z_y); lse - z_y and
// p_y - 1 would cancel for a confident prediction.  dz is kept in units of the largest finite weight of the piece, which the
// epilogues of (2) and (3) multiply in fp32.
//
// The tensor cores cut off what does not fit into their running sum, towards zero, so a sum of many products comes out short.  By
// how much depends on the values; measured, in units of 2^-30 of the sum per nonzero feature of x: normal values 0.83 to 1.07
// (256 to 65536 features), half or nine tenths of the features zero 1.5, nine tenths of 65536 3.2, products of one sign 4 to 6, a few
// features a hundred times the others 2 where they come first and 0.04 where they come last, one to four features and small whole
// numbers none.
// The logits of a row are therefore scaled up by 1 + 2^-30 n with n its nonzero features (lm_rows_kernel).  For 4096 normal
// values that halves a logit's error (4.4e-6 -> 2.2e-6 of the logits' size) and takes most of lse's, where nearly equal shares add
// up (3.9e-6 -> 5e-7); a row of up to 64 features is left as it is, and a dense row that lost nothing is off by 2^-30 n of its
// logits.  dx and dw round to bf16.
//
// Products: persistent, K in blocks of 64 (128-byte-swizzled TMA boxes), a four-stage ring of 48 KiB stages:
//   warp 0      TMA producer
//   warp 1      tcgen05.mma issuer, two 256-column accumulators in TMEM
//   warps 2-9   epilogue (a thread owns a row of an accumulator)
// Tiles of 128 x 256 by single CTAs, or of 512 x 256 by pairs (see lm_gemm_kernel).  W and x are read as they lie: K-major for (1),
// as MN-major operands for (2) and (3); dz K-major for (2) and MN-major for (3); nothing is transposed in memory.
//
// Rows of all ranks are put together in slots of 8..128 rows (a power of two, by the rows of a rank), so that a tile holds several
// ranks where a rank has few tokens.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include <atomic>

#include "common.cuh"
#include "ptx.cuh"
#include "spans.h"
#include "tmap.cuh"

int *basp_status_device_ptr();

namespace {

using namespace ptx;

constexpr int kBM = 128, kBN = 256, kBK = 64;      // rows of an accumulator, columns of a tile, K block
constexpr int kABytes = kBM * kBK * 2;
template <bool kPair>
constexpr int kRowsPerCta = kPair ? 2 * kBM : kBM;
template <bool kPair>
constexpr int kTileM = kPair ? 4 * kBM : kBM;
constexpr int kThreads = 320;                      // TMA warp, MMA warp, eight epilogue warps
constexpr int kStagingBytes = 4 << 10;             // of an epilogue warp: 32 rows of 128 bytes
constexpr int kStages = 4, kStageBytes = 48 << 10; // A 128 and B 256 rows of 128 bytes, or A 256 and half of B
constexpr int kMnBlock = kBK * 64 * 2;             // one 64-column block of an MN-major operand: 64 rows of 128 bytes
constexpr int kSms = 148;                          // of the GPU this code is written for; plans the split, not the grid
constexpr int kStatCols = 128;                     // columns that share a maximum: as many as a thread holds in registers
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kCodeStep = 1024.f;                // distances in 2^-10 of log2
constexpr float kCodeMax = 65535.f;                // and above: probability zero

enum Kind { kStats = 0, kLogits = 1, kDx = 2, kDw = 3 };

// Which token a row of the piece is.
struct Rows {
    int slot_log2;             // rows per slot
    int slot_begin, slots;     // the piece's slots
    int per_rank;              // slots per rank
    int K, M, M_last;          // ranks per group; rows of a rank, and of a group's last rank
};
struct Token {
    int rank, row;
    bool valid;
};
__device__ __forceinline__ Token token_of(const Rows &s, int i) {
    Token t;
    const int slot = i >> s.slot_log2, at = s.slot_begin + slot;
    t.rank = at / s.per_rank;
    t.row = ((at - t.rank * s.per_rank) << s.slot_log2) + (i & ((1 << s.slot_log2) - 1));
    t.valid = slot < s.slots && t.row < (t.rank % s.K == s.K - 1 ? s.M_last : s.M);
    return t;
}

template <int R>
struct LossParams {
    CUtensorMap x[R];          // (1): boxes of one slot
    CUtensorMap w, dz;
    CUtensorMap dw;            // (3): boxes of a warp's 32 rows
    CUtensorMap kept;          // (3): the piece's rows of x, zero where a row has no part in the gradients
    const long long *label[R];
    __nv_bfloat16 *dx[R];
    Rows rows;
    int tiles_m, tiles_n, k_blocks, splits, group;
    int vocab, hidden;
    const float *cut;          // (1): what the products of each row cut off, as a share of the sum
    bool wide;                 // (2): every row of the result starts on a multiple of 32 bytes
    size_t pitch;              // columns of a row of 16-bit logits
    int piece_rows;
    float2 *stats;             // [groups of kStatCols columns][piece_rows]: maximum as the products left it, sum
    unsigned *scale;           // bits of the largest finite |weight| of the piece: dz is in its units, so that equal weights leave
                               // p - 1 as it is (rounding -1 g would be one relative error common to all tokens)
    uint16_t *codes;           // [piece_rows][pitch]
    float *partial;            // (2) with splits > 1: [splits][partial_rows][hidden]
    int partial_rows;          // the rows of this piece, which may be fewer than piece_rows
    const float *acc_in;       // (3) sum of the earlier pieces, or NULL
    float *acc_out;            // (3) sum so far, or NULL: the result
    int *status;
};

struct Bars {
    uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort_flag;
};

#define LOSS_WAIT(bar, parity, role, detail)                                    \
    do {                                                                        \
        if (!mbar_wait((bar), (parity), &bars.abort_flag)) {                   \
            bars.abort_flag = 1;                                                \
            if (atomicCAS(p.status, 0, 6) == 0) {                               \
                p.status[1] = (role); p.status[2] = (int)blockIdx.x; p.status[3] = (detail); \
            }                                                                   \
            goto gemm_done;                                                     \
        }                                                                       \
    } while (0)

// Tile coordinates of a work item: row tiles in groups, within a group row tiles fastest.  The SMs work on neighbouring
// items at the same time, so a group's first operand stays in L2 while the second streams by.
struct Item {
    int m, n, kb0, kb1;
    int split;
};
template <int kKind, int R>
__device__ __forceinline__ Item item_of(const LossParams<R> &p, int i) {
    Item t;
    t.split = 0; t.kb0 = 0; t.kb1 = p.k_blocks;
    if constexpr (kKind == kDx) {
        const int tiles = p.tiles_m * p.tiles_n;
        t.split = i / tiles;
        i -= t.split * tiles;
        t.kb0 = (int)((long long)p.k_blocks * t.split / p.splits);
        t.kb1 = (int)((long long)p.k_blocks * (t.split + 1) / p.splits);
    }
    const int per_group = p.group * p.tiles_n, g = i / per_group, m0 = g * p.group;
    const int wide = min(p.group, p.tiles_m - m0);
    i -= g * per_group;
    t.n = i / wide;
    t.m = m0 + i - t.n * wide;
    return t;
}

// 32 columns of a row, or its last `cols` (a multiple of 8).  wide: rows start on multiples of 32 bytes, whole sectors at a time
__device__ __forceinline__ void store_bf16x32(__nv_bfloat16 *dst, const float (&v)[32], int cols, bool wide) {
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    if (wide) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (16 * i < cols)
                asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                             :: "l"(dst + 16 * i), "r"(w[8 * i]), "r"(w[8 * i + 1]), "r"(w[8 * i + 2]), "r"(w[8 * i + 3]),
                                "r"(w[8 * i + 4]), "r"(w[8 * i + 5]), "r"(w[8 * i + 6]), "r"(w[8 * i + 7]) : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (8 * i < cols) *reinterpret_cast<uint4 *>(dst + 8 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
}

// kPair = false: a CTA works on 128 x 256 tiles; its two accumulators take turns, so that the epilogue of one tile runs under the
// main loop of the next.
// kPair = true: two neighbouring CTAs (a cluster) work on one 512 x 256 tile, each with 256 of its rows and half of B, so that a
// product needs half the bytes from L2; the two accumulators of a CTA are the upper and lower 128 of its rows.  The last blocks of
// K are issued for the upper rows first, the first blocks of the next tile too: either epilogue then runs under the other half's
// products.
template <int kKind, int R, bool kPair>
__global__ void __launch_bounds__(kThreads, 1) lm_gemm_kernel(const __grid_constant__ LossParams<R> p) {
    constexpr int kS = kStages, kRows = kRowsPerCta<kPair>, kBCols = kPair ? kBN / 2 : kBN;
    constexpr int kA = kRows * kBK * 2, kB = kBCols * kBK * 2;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sA = smem;
    uint8_t *sB = smem + kS * kA;
    __shared__ Bars bars;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int total = p.tiles_m * p.tiles_n * p.splits;
    const int half = kPair ? (int)cluster_rank() : 0;      // this CTA's rows and columns of the tile
    const int first = kPair ? blockIdx.x >> 1 : blockIdx.x, step = kPair ? gridDim.x >> 1 : gridDim.x;

    if (tid == 0) {
        for (int s = 0; s < kS; ++s) { mbar_init(&bars.full[s], 1); mbar_init(&bars.empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&bars.acc_full[a], 1); mbar_init(&bars.acc_empty[a], 8); }
        bars.abort_flag = 0;
        fence_mbar_init();
        if (kKind == kLogits && blockIdx.x == 0) *p.scale = 0;
    }
    if (warp == 1) {
        if constexpr (kPair) { tmem_alloc_pair(&bars.tmem_base, 512); tmem_relinquish_pair(); }
        else { tmem_alloc(&bars.tmem_base, 512); tmem_relinquish(); }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (kPair) cluster_sync();                   // both CTAs' barriers and tensor memory are there
    tc_fence_after();
    const uint32_t tmem = bars.tmem_base;
    allow_next_kernel();                                   // the pass behind this product has work of its own to start with

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer (lane 0 issues)
        uint32_t it = 0;
        for (int i = first; i < total; i += step) {
            const Item t = item_of<kKind>(p, i);
            const int m0 = t.m * kTileM<kPair> + half * kRows, n0 = t.n * kBN + half * kBCols;
            int mine = 0;                                  // (1): slots of this CTA's rows
            uint32_t expect = (kA + kB) * (kPair ? 2 : 1); // bytes of the tile's K block
            if constexpr (kKind == kStats || kKind == kLogits) {
                const int per_cta = kRows >> p.rows.slot_log2, rest = p.rows.slots - t.m * (kTileM<kPair> >> p.rows.slot_log2);
                mine = min(per_cta, max(0, rest - half * per_cta));
                expect = kB * (kPair ? 2 : 1) + (uint32_t)(min(rest, kPair ? 2 * per_cta : per_cta) << p.rows.slot_log2) * kBK * 2;
            }
            for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
                const uint32_t s = it % kS, ph = (it / kS) & 1;
                LOSS_WAIT(&bars.empty[s], ph ^ 1, 0, kb);
                if (lane == 0) {
                    uint8_t *a = sA + s * kA, *b = sB + s * kB;
                    // a pair's loads are all counted on the first CTA's barrier
                    const uint32_t bar = kPair ? map_to_rank(&bars.full[s], 0) : 0;
                    if (half == 0) mbar_arrive_expect_tx(&bars.full[s], expect);
                    auto load = [&](uint8_t *dst, const CUtensorMap *map, int c, int r) {
                        if constexpr (kPair) tma_load_3d_pair(dst, map, bar, c, 0, r);
                        else tma_load_3d(dst, map, &bars.full[s], c, 0, r);
                    };
                    if constexpr (kKind == kStats || kKind == kLogits) {
                        // W, which comes from HBM, is asked for before x (1 token: 1.1 us of 30)
                        load(b, &p.w, kb * kBK, n0);
                        // slots past the piece's end are left as they are: a row of A reaches its own row of the product only
                        for (int j = 0; j < mine; ++j) {
                            const int at = p.rows.slot_begin + (m0 >> p.rows.slot_log2) + j, r = at / p.rows.per_rank;
                            load(a + (j << p.rows.slot_log2) * kBK * 2, &p.x[r], kb * kBK, (at - r * p.rows.per_rank) << p.rows.slot_log2);
                        }
                    } else if constexpr (kKind == kDx) {
#pragma unroll
                        for (int j = 0; j < kRows; j += kBM) load(a + j * kBK * 2, &p.dz, kb * kBK, m0 + j);
#pragma unroll
                        for (int c = 0; c < kBCols / 64; ++c) load(b + c * kMnBlock, &p.w, n0 + c * 64, kb * kBK);
                    } else {
#pragma unroll
                        for (int c = 0; c < kRows / 64; ++c) load(a + c * kMnBlock, &p.dz, m0 + c * 64, kb * kBK);
#pragma unroll
                        for (int c = 0; c < kBCols / 64; ++c) load(b + c * kMnBlock, &p.kept, n0 + c * 64, kb * kBK);
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (lane 0 of the first CTA issues)
        const uint32_t idesc = make_idesc_bf16(kPair ? 2 * kBM : kBM, kBN, kKind == kDw, kKind == kDx || kKind == kDw);
        const uint64_t desc_k = make_smem_desc_sw128(0, 16, 1024), desc_mn = make_smem_desc_sw128(0, kMnBlock, 1024);
        const uint64_t da0 = (kKind == kDw ? desc_mn : desc_k) | (uint64_t)(smem_u32(sA) >> 4);
        const uint64_t db0 = (kKind == kDx || kKind == kDw ? desc_mn : desc_k) | (uint64_t)(smem_u32(sB) >> 4);
        // 16 elements of K: 32 bytes along a row, or 16 rows of 128 bytes
        constexpr int kStepA = kKind == kDw ? 128 : 2, kStepB = kKind == kDx || kKind == kDw ? 128 : 2;
        // 128 rows (of each CTA) from `sub` on, stage s, into accumulator acc
        auto products = [&](uint32_t s, int sub, uint32_t acc, bool fresh) {
            if (lane != 0) return;
            const uint64_t da = da0 + s * (kA >> 4) + sub * (kABytes >> 4), db = db0 + s * (kB >> 4);
#pragma unroll
            for (int kk = 0; kk < kBK / 16; ++kk) {
                if constexpr (kPair)
                    mma_ss_pair(tmem + acc * kBN, da + kk * kStepA, db + kk * kStepB, idesc, !fresh || (kk > 0));
                else
                    mma_ss(tmem + acc * kBN, da + kk * kStepA, db + kk * kStepB, idesc, !fresh || (kk > 0));
            }
        };
        auto commit = [&](uint64_t *bar) {
            if (lane != 0) return;
            if constexpr (kPair) tc_commit_pair(bar);
            else tc_commit(bar);
        };
        uint32_t it = 0, cnt = 0;
        for (int i = half == 0 ? first : total; i < total; i += step, ++cnt) {
            const Item t = item_of<kKind>(p, i);
            const int n = t.kb1 - t.kb0;
            if constexpr (!kPair) {
                const uint32_t acc = cnt & 1;
                LOSS_WAIT(&bars.acc_empty[acc], ((cnt >> 1) & 1) ^ 1, 1, i);
                tc_fence_after();
                for (int u = 0; u < n; ++u, ++it) {
                    const uint32_t s = it % kS;
                    LOSS_WAIT(&bars.full[s], (it / kS) & 1, 2, u);
                    tc_fence_after();
                    products(s, 0, acc, u == 0);
                    commit(&bars.empty[s]);
                }
                commit(&bars.acc_full[acc]);
            } else {
                const int head = min(kS, n), tail = min(kS, n - head);
                LOSS_WAIT(&bars.acc_empty[0], (cnt & 1) ^ 1, 1, i);
                tc_fence_after();
                for (int u = 0; u < head; ++u) {
                    const uint32_t s = (it + u) % kS;
                    LOSS_WAIT(&bars.full[s], ((it + u) / kS) & 1, 2, u);
                    tc_fence_after();
                    products(s, 0, 0, u == 0);
                }
                if (tail == 0) commit(&bars.acc_full[0]);
                LOSS_WAIT(&bars.acc_empty[1], (cnt & 1) ^ 1, 1, i);
                tc_fence_after();
                for (int u = 0; u < head; ++u, ++it) {
                    products(it % kS, 1, 1, u == 0);
                    commit(&bars.empty[it % kS]);
                }
                for (int u = head; u < n - tail; ++u, ++it) {
                    const uint32_t s = it % kS;
                    LOSS_WAIT(&bars.full[s], (it / kS) & 1, 2, u);
                    tc_fence_after();
                    products(s, 0, 0, false);
                    products(s, 1, 1, false);
                    commit(&bars.empty[s]);
                }
                for (int u = 0; u < tail; ++u) {
                    const uint32_t s = (it + u) % kS;
                    LOSS_WAIT(&bars.full[s], ((it + u) / kS) & 1, 2, u);
                    tc_fence_after();
                    products(s, 0, 0, false);
                }
                if (tail > 0) commit(&bars.acc_full[0]);
                for (int u = 0; u < tail; ++u, ++it) {
                    products(it % kS, 1, 1, false);
                    commit(&bars.empty[it % kS]);
                }
                commit(&bars.acc_full[1]);
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue (the other warps)
        const int quarter = warp & 3;                       // the TMEM lanes this warp can reach
        const int row = quarter * 32 + lane;
        const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
        if constexpr (kKind == kStats || kKind == kLogits) wait_previous_kernel();         // what `cut` comes from; the operands do not
        uint8_t *staging = smem + kStages * kStageBytes + (warp - 2) * kStagingBytes;       // (3)
        uint32_t cnt = 0;
        float scale = 1.f;
        if constexpr (kKind == kDx || kKind == kDw) scale = __uint_as_float(*p.scale);
        for (int i = first; i < total; i += step, ++cnt) {
            const Item t = item_of<kKind>(p, i);
            const uint32_t acc = kPair ? (warp - 2) >> 2 : cnt & 1, parity = kPair ? cnt & 1 : (cnt >> 1) & 1;
            // a pair's warp takes all columns of its accumulator, a single CTA's four warps each take half of them
            constexpr int kCols = kPair ? kBN : kBN / 2;
            const int side = kPair ? 0 : ((warp - 2) >> 2) * kCols;
            const uint32_t src = tmem + acc * kBN + side + lane_addr;
            const int prow = t.m * kTileM<kPair> + half * kRows + (kPair ? acc * kBM : 0) + row;
            auto hand_back = [&] {                          // the accumulator is in registers
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (kPair) mbar_arrive_at(map_to_rank(&bars.acc_empty[acc], 0));
                    else mbar_arrive(&bars.acc_empty[acc]);
                }
            };
            const int col0 = t.n * kBN + side;
            if constexpr (kKind == kStats || kKind == kLogits) {
                const Token tok = token_of(p.rows, prow);
                const long long label = tok.valid ? p.label[tok.rank][tok.row] : -1;
                // the target's column in this tile, or -1
                const int hit = label >= col0 && label < p.vocab && label < col0 + kCols ? (int)(label - col0) : -1;
                const bool stored = prow < p.piece_rows;            // not the second half of an odd last tile
                const float unit = fmaf(kLog2e, stored ? p.cut[prow] : 0.f, kLog2e);       // of a distance
                LOSS_WAIT(&bars.acc_full[acc], parity, 3, i);
                tc_fence_after();
                uint16_t *dst = p.codes + (size_t)prow * p.pitch + col0;
#pragma unroll 1
                for (int g = 0; g < kCols / kStatCols; ++g) {
                    uint32_t v[kStatCols / 32][32];
#pragma unroll
                    for (int c = 0; c < kStatCols / 32; ++c) tmem_ld_x32(src + g * kStatCols + c * 32, v[c]);
                    tmem_wait_ld();
                    if (g == kCols / kStatCols - 1) hand_back();
                    // columns that do not count (the target, columns past the vocabulary) become -inf
                    const int at = hit - g * kStatCols, cols = p.vocab - col0 - g * kStatCols;
                    if (__any_sync(0xffffffffu, (at >= 0 && at < kStatCols) || cols < kStatCols)) {
#pragma unroll
                        for (int c = 0; c < kStatCols / 32; ++c)
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (c * 32 + e == at || c * 32 + e >= cols) v[c][e] = 0xff800000u;
                    }
                    float m = -INFINITY;
#pragma unroll
                    for (int c = 0; c < kStatCols / 32; ++c)
#pragma unroll
                        for (int e = 0; e < 32; e += 2) m = max3(m, __uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1]));
                    // Distances are differences first and scaled after: zero for the largest itself and below zero for all others,
                    // however far from zero the logits lie (v log2e - m log2e in one operation would be off by the rounding of
                    // m log2e, to either side).  Nothing but the target: distances are infinite
                    const float base = m == -INFINITY ? 0.f : -m;
                    const uint64_t base2 = pack_f2(base, base), unit2 = pack_f2(unit, unit);
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < kStatCols / 32; ++c) {
                        uint32_t out[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float d[2];            // log2 of the terms, <= 0
                            unpack_f2(mul2(add2(pack_f2(__uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1])), base2), unit2), d[0], d[1]);
                            sum[e & 3] += exp2_approx(d[0]);
                            sum[(e & 3) + 1] += exp2_approx(d[1]);
                            if constexpr (kKind == kLogits) {
                                // + 2^23: the nearest whole number in the low bits
                                uint32_t code[2];
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    code[h] = __float_as_uint(fminf(fmaf(d[h], -kCodeStep, 8388608.f), 8388608.f + kCodeMax));
                                out[e / 2] = __byte_perm(code[0], code[1], 0x5410);
                            }
                        }
                        if constexpr (kKind == kLogits) {
                            if (stored) {
#pragma unroll
                                for (int q = 0; q < 4; ++q)
                                    *reinterpret_cast<uint4 *>(dst + g * kStatCols + c * 32 + 8 * q) =
                                        make_uint4(out[4 * q], out[4 * q + 1], out[4 * q + 2], out[4 * q + 3]);
                            }
                        }
                    }
                    if (stored)
                        p.stats[(size_t)(col0 / kStatCols + g) * p.piece_rows + prow] =
                            make_float2(m, (sum[0] + sum[1]) + (sum[2] + sum[3]));
                }
            } else {
                const int width = min(kCols, p.hidden - col0);      // a multiple of 8
                Token tok{0, prow, prow < p.vocab};
                if constexpr (kKind == kDx) tok = token_of(p.rows, prow);
                LOSS_WAIT(&bars.acc_full[acc], parity, 3, i);
                tc_fence_after();
                for (int c = 0; c < kCols / 32; ++c) {
                    uint32_t raw[32];
                    tmem_ld_x32(src + c * 32, raw);
                    tmem_wait_ld();
                    if (c == kCols / 32 - 1) hand_back();
                    const int cols = min(32, width - c * 32);
                    const bool live = tok.valid && cols > 0;
                    float v[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(raw[e]) * scale;
                    if constexpr (kKind == kDx) {
                        if (!live) continue;
                        if (p.splits == 1) {
                            store_bf16x32(p.dx[tok.rank] + (size_t)tok.row * p.hidden + col0 + c * 32, v, cols, p.wide);
                        } else {
                            float *dst = p.partial + ((size_t)t.split * p.partial_rows + prow) * p.hidden + col0 + c * 32;
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                if (4 * q < cols) *reinterpret_cast<float4 *>(dst + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                        }
                    } else {
                        const size_t at = (size_t)prow * p.hidden + col0 + c * 32;
                        if (p.acc_in && live) {
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                if (4 * q < cols) {
                                    const float4 o = *reinterpret_cast<const float4 *>(p.acc_in + at + 4 * q);
                                    v[4 * q] += o.x; v[4 * q + 1] += o.y; v[4 * q + 2] += o.z; v[4 * q + 3] += o.w;
                                }
                        }
                        if (p.acc_out) {
                            if (!live) continue;
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                if (4 * q < cols) *reinterpret_cast<float4 *>(p.acc_out + at + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                        } else {
                            // 64 columns of the warp's 32 rows at a time through shared memory: stored by lanes, each in a row of
                            // its own, they keep the load/store unit busy for one line per lane (dW of 48 tokens: 68 us)
                            if (c % 2 == 0) {
                                if (lane == 0) tma_store_wait_read<0>();
                                __syncwarp();
                            }
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                *reinterpret_cast<uint4 *>(staging + lane * 128 + ((((c & 1) * 4 + q) ^ (lane & 7)) << 4)) =
                                    make_uint4(pack_bf16x2(v[8 * q], v[8 * q + 1]), pack_bf16x2(v[8 * q + 2], v[8 * q + 3]),
                                               pack_bf16x2(v[8 * q + 4], v[8 * q + 5]), pack_bf16x2(v[8 * q + 6], v[8 * q + 7]));
                            if (c % 2 == 1) {
                                fence_proxy_async_smem();
                                __syncwarp();
                                const int first_col = col0 + (c - 1) * 32, first_row = prow - lane;
                                if (lane == 0 && first_col < p.hidden && first_row < p.vocab) {     // the ends are cut off by the copy
                                    tma_store_3d(&p.dw, staging, first_col, 0, first_row);
                                    tma_store_commit();
                                }
                            }
                        }
                    }
                }
            }
        }
        if (kKind == kDw && lane == 0) tma_store_wait<0>();
    }

gemm_done:
    tc_fence_before();
    __syncthreads();
    if (bars.abort_flag) {
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) { }
        __syncthreads();
    }
    if constexpr (kPair) cluster_sync();                   // the other CTA may still signal this one's barriers
    if (warp == 1) {
        if constexpr (kPair) tmem_dealloc_pair(tmem, 512);
        else tmem_dealloc(tmem, 512);
    }
}

#undef LOSS_WAIT

// ------------------------------------------------------------------------------------------------ statistics of the rows
struct RowInfo {               // what the element-wise pass needs of a row
    float top, rest;           // lse = top (1 + cut) + rest, top: the largest logit besides the target's, as the products left it.  One
                               // number would be off by its rounding, an error of every probability where logits are large
    float unit;                // of a distance of two logits in log2, with what the products cut off
    float weight, target_dz;   // target_dz: without the weight
    int label;                 // -1: none
};

template <int R>
struct MergeParams {
    const long long *label[R];
    const float *weight[R];    // a NULL table entry: weight 1
    const __nv_bfloat16 *x[R], *w;
    float *loss[R], *lse[R];
    Rows rows;
    int groups, piece_rows, vocab, hidden;
    const float2 *stats;
    const float *cut;
    unsigned *scale;
    RowInfo *info;             // NULL: not wanted
};

// `unit`: of a distance in log2
__device__ __forceinline__ void join(float &m, float &s, float m2, float s2, float unit) {
    const float top = fmaxf(m, m2), use = top == -INFINITY ? 0.f : top;
    s = s * exp2f((m - use) * unit) + s2 * exp2f((m2 - use) * unit);
    m = top;
}

// What the products with a row cut off, as a share of the sums.  A warp takes a row.
template <int R>
struct CutParams {
    const __nv_bfloat16 *x[R];
    Rows rows;
    int hidden;
    float *cut;
};
template <int R>
__global__ void __launch_bounds__(256) lm_rows_kernel(const __grid_constant__ CutParams<R> p) {
    const int lane = threadIdx.x & 31, row = blockIdx.x * 8 + (threadIdx.x >> 5);
    allow_next_kernel();
    const Token tok = token_of(p.rows, row);
    int n = 0;
    if (tok.valid) {
        const uint4 *x = reinterpret_cast<const uint4 *>(p.x[tok.rank] + (size_t)tok.row * p.hidden);
#pragma unroll 8
        for (int c = lane; c < p.hidden / 8; c += 32) {
            const uint4 u = __ldg(x + c);
            const uint32_t us[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) n += ((us[q] & 0x7fffu) != 0) + ((us[q] & 0x7fff0000u) != 0);
        }
    }
    n = __reduce_add_sync(0xffffffffu, n);
    // 64 features: 2^-24, which a sum loses in its own rounding
    if (lane == 0) p.cut[row] = n > 64 ? (float)n * 0x1p-30f : 0.f;
}

// A block takes 32 rows.  Its 32 warps share the column groups (neighbouring lanes read neighbouring rows), then each takes one
// row: the target's logit, the join of the warps' sums, the loss.
template <int R>
__global__ void __launch_bounds__(1024) lm_merge_kernel(const __grid_constant__ MergeParams<R> p) {
    __shared__ float2 part[32][33];
    __shared__ unsigned scale;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) scale = 0;
    const int row = blockIdx.x * 32 + warp;
    const Token tok = token_of(p.rows, row);
    const long long label = tok.valid ? p.label[tok.rank][tok.row] : -1;
    const bool counts = label >= 0 && label < p.vocab;
    // the target's logit in fp32 operations rounded to nearest: the tensor cores' sum of a large logit (they cut off what does
    // not fit) would be the largest error of the loss
    float z = 0.f;
    if (counts) {
        const uint4 *x = reinterpret_cast<const uint4 *>(p.x[tok.rank] + (size_t)tok.row * p.hidden);
        const uint4 *w = reinterpret_cast<const uint4 *>(p.w + (size_t)label * p.hidden);
        float a[8] = {};
#pragma unroll 8
        for (int c = lane; c < p.hidden / 8; c += 32) {
            const uint4 u = __ldg(x + c), v = __ldg(w + c);
            const uint32_t us[4] = {u.x, u.y, u.z, u.w}, vs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                a[2 * q] = fmaf(__uint_as_float(us[q] << 16), __uint_as_float(vs[q] << 16), a[2 * q]);
                a[2 * q + 1] = fmaf(__uint_as_float(us[q] & 0xffff0000u), __uint_as_float(vs[q] & 0xffff0000u), a[2 * q + 1]);
            }
        }
        z = ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
    }
    wait_previous_kernel();                        // up to here only the call's inputs were read
    {
        const int i = blockIdx.x * 32 + lane;
        float m = -INFINITY, s = 0.f;
        const float unit = fmaf(kLog2e, p.cut[i], kLog2e);
        constexpr int kBatch = 8;                  // loads in flight
        for (int n0 = warp; n0 < p.groups; n0 += 32 * kBatch) {
            float2 v[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int n = n0 + 32 * u;
                v[u] = n < p.groups ? p.stats[(size_t)n * p.piece_rows + i] : make_float2(-INFINITY, 0.f);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) join(m, s, v[u].x, v[u].y, unit);
        }
        part[warp][lane] = make_float2(m, s);
    }
    __syncthreads();
    const float2 mine = part[lane][warp];
    float m = mine.x, s = 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        z += __shfl_xor_sync(0xffffffffu, z, o);
    }
    const float cut = p.cut[row], unit = fmaf(kLog2e, cut, kLog2e);
    s = mine.y * exp2f((mine.x - (m == -INFINITY ? 0.f : m)) * unit);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) {
        RowInfo info{0.f, 0.f, unit, 0.f, 0.f, -1};
        if (tok.valid) {
            info.top = m == -INFINITY ? 0.f : m;
            // lse - top; `back`: of that, what the products cut off top itself
            const float back = info.top * cut;
            float loss = 0.f, rest = logf(s) + back;       // -inf where the target is the only word
            if (counts) {
                // differences of logits first: they stay small where the logits are large
                const float away = (info.top - z) + rest, tail = log1pf(expf(-fabsf(away)));
                loss = (away > 0.f ? away : 0.f) + tail;
                rest = (away > 0.f ? rest : z - info.top) + tail;
                if (p.info) {
                    info.weight = p.weight[tok.rank] ? p.weight[tok.rank][tok.row] : 1.f;
                    info.target_dz = -1.f / (1.f + expf(-away));
                    info.label = (int)label;
                }
            }
            info.rest = rest - back;
            p.loss[tok.rank][tok.row] = loss;
            if (p.lse[tok.rank]) p.lse[tok.rank][tok.row] = info.top + rest;
        }
        if (p.info) {
            p.info[row] = info;
            // a weight that is no finite number is not a unit: it reaches its own dx and dw, not other tokens' dx
            const float size = fabsf(info.weight);
            atomicMax(&scale, size < INFINITY ? __float_as_uint(size) : 0u);
        }
    }
    if (!p.info) return;
    __syncthreads();
    if (threadIdx.x == 0) atomicMax(p.scale, scale);
}

// ------------------------------------------------------------------------------------------------ 16-bit distances -> bf16 dz
// In place.  A warp takes 256 columns of one row at a time (two column groups), a lane 8 columns.  A row
// without weight is written as zeros and not read: nothing of it, NaN neither, reaches the gradients.  The row's last block
// copies x.
constexpr int kDzTiles = 4;    // tiles per warp
template <int R>
struct DzParams {
    const __nv_bfloat16 *x[R];
    Rows rows;
    __nv_bfloat16 *kept;       // [piece_rows][hidden], or NULL
    uint16_t *codes;
    size_t pitch;
    const RowInfo *info;
    const float2 *stats;
    const unsigned *scale;
    int tiles_n, piece_rows, hidden, blocks;       // blocks: of a row's logits
};
template <int R>
__global__ void __launch_bounds__(256) lm_dz_kernel(const __grid_constant__ DzParams<R> p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.y;
    const RowInfo info = p.info[row];
    if ((int)blockIdx.x == p.blocks) {
        const Token tok = token_of(p.rows, row);
        const bool read = tok.valid && info.weight != 0.f;
        const uint4 *src = reinterpret_cast<const uint4 *>(read ? p.x[tok.rank] + (size_t)tok.row * p.hidden : nullptr);
        uint4 *dst = reinterpret_cast<uint4 *>(p.kept + (size_t)row * p.hidden);
#pragma unroll 4
        for (int i = threadIdx.x; i < p.hidden / 8; i += 256) dst[i] = read ? __ldg(src + i) : make_uint4(0, 0, 0, 0);
        return;
    }
    const int tiles_n = p.tiles_n, piece_rows = p.piece_rows;
    const float weight = __fdiv_rn(info.weight, __uint_as_float(*p.scale));     // exactly 1 where all are equal
    const int n0 = (blockIdx.x * 8 + warp) * kDzTiles;
    uint4 v[kDzTiles];
    float m[kDzTiles];
    uint4 *at = reinterpret_cast<uint4 *>(p.codes + (size_t)row * p.pitch) + (size_t)n0 * 32 + lane;
    if (info.weight != 0.f) {
#pragma unroll
        for (int u = 0; u < kDzTiles; ++u)
            if (n0 + u < tiles_n) {
                v[u] = at[u * 32];
                m[u] = __ldg(&p.stats[(size_t)((n0 + u) * (kBN / kStatCols) + lane / (kStatCols / 8)) * piece_rows + row].x);
            }
    }
#pragma unroll
    for (int u = 0; u < kDzTiles; ++u) {
        if (n0 + u >= tiles_n) break;
        uint4 o = make_uint4(0, 0, 0, 0);
        if (info.weight != 0.f) {
            const float c = (m[u] - info.top) * info.unit - info.rest * kLog2e;
            const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
            const int target = info.label - ((n0 + u) * 256 + lane * 8);
            uint32_t r[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float d[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t code = e ? w[q] >> 16 : w[q] & 0xffffu;
                    const float dist = code == 65535u ? INFINITY : (float)code * (1.f / kCodeStep);
                    d[e] = (2 * q + e == target ? info.target_dz : exp2_approx(c - dist)) * weight;
                }
                r[q] = pack_bf16x2(d[0], d[1]);
            }
            o = make_uint4(r[0], r[1], r[2], r[3]);
        }
        at[u * 32] = o;
    }
}

// ------------------------------------------------------------------------------------------------ dx from its partial sums
template <int R>
struct JoinParams {
    __nv_bfloat16 *dx[R];
    Rows rows;
    const float *partial;
    int splits, partial_rows, hidden;
};
template <int R>
__global__ void __launch_bounds__(256) lm_dx_join_kernel(const __grid_constant__ JoinParams<R> p) {
    const int per_row = p.hidden / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(i / per_row), c = (int)(i - (long long)row * per_row) * 8;
    wait_previous_kernel();
    if (row >= p.partial_rows) return;
    const Token tok = token_of(p.rows, row);
    if (!tok.valid) return;
    float s[8] = {};
    for (int k = 0; k < p.splits; ++k) {
        const float4 *src = reinterpret_cast<const float4 *>(p.partial + ((size_t)k * p.partial_rows + row) * p.hidden + c);
        const float4 a = src[0], b = src[1];
        s[0] += a.x; s[1] += a.y; s[2] += a.z; s[3] += a.w; s[4] += b.x; s[5] += b.y; s[6] += b.z; s[7] += b.w;
    }
    uint4 o;
    o.x = pack_bf16x2(s[0], s[1]); o.y = pack_bf16x2(s[2], s[3]); o.z = pack_bf16x2(s[4], s[5]); o.w = pack_bf16x2(s[6], s[7]);
    *reinterpret_cast<uint4 *>(p.dx[tok.rank] + (size_t)tok.row * p.hidden + c) = o;
}

// ------------------------------------------------------------------------------------------------ host side
constexpr int kDefaultPiece = 8192, kMaxPiece = 32768, kMaxDevices = 64;
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
int cdiv(long long a, long long b) { return (int)((a + b - 1) / b); }

// Sizes of one call: slots, pieces, and the workspace.
struct Sizes {
    int slot_log2, per_rank, slots;                // slots of all ranks
    int tiles_m, piece_tiles, pieces;              // row tiles in all and per piece
    int tiles_v, tiles_h;                          // 256-column tiles of the vocabulary and of `hidden`
    size_t pitch;
};

// A pair's tile takes 0.85 of the time of four single CTAs' tiles (1024 rows of 4096 against 128256 words: 855 and 894 us; 512:
// 406 and 472; under the power limit its fewer bytes from L2, 24 instead of 48 KiB per 128 x 256 x 64 products, count for more),
// but it is 512 rows high: for 320 rows a single CTA's three tiles are faster (359 and 380 us), for 768 its six (705 and 787).
bool use_pair(int rows) { return 0.85 * 4 * cdiv(rows, kTileM<true>) < cdiv(rows, kTileM<false>); }

// How often the vocabulary is split in dx = dz W: the time of `waves` rounds of tiles over the SMs, a tile costing its K
// blocks plus a start and an epilogue (8 blocks), plus writing and reading the partial sums.
int dx_splits(int tiles_m, int tiles_h, int k_blocks, int hidden) {
    const double block_us = 0.43;                  // 128 x 256 x 64 at the sustained rate of one SM
    const bool pair = use_pair(tiles_m * kBM);
    int best = 1;
    double best_us = 1e30;
    for (int s = 1; s <= 64 && (s == 1 || k_blocks / s >= 8); ++s) {
        const double bytes = (double)s * tiles_m * kBM * hidden * 4;
        if (s > 1 && bytes > 768e6) break;
        // rounds of items over SMs or pairs; a pair's block is four times the work of two SMs
        const double us = (double)(pair ? cdiv((long long)cdiv(tiles_m, 4) * tiles_h * s, kSms / 2)
                                        : cdiv((long long)tiles_m * tiles_h * s, kSms)) *
                              (cdiv(k_blocks, s) + 8) * (pair ? 2 * block_us : block_us) +
                          (s > 1 ? 4.0 + 2 * bytes / 6.0e6 : 0.0);
        if (us < best_us) { best_us = us; best = s; }
    }
    return best;
}

int sizes_of(const basp_plan *p, int hidden, int vocab, int piece_rows, Sizes *z) {
    if (hidden <= 0 || vocab <= 0 || piece_rows < 0) return BASP_ERR_INVALID;
    if (hidden % 8 != 0 || hidden > 65536 || vocab > (1 << 24) || piece_rows > kMaxPiece) return BASP_ERR_UNSUPPORTED;
    const long long M = (long long)p->Bl * p->T;
    if (M * p->N >= (1ll << 30)) return BASP_ERR_UNSUPPORTED;
    z->slot_log2 = 3;
    while (z->slot_log2 < 7 && (1ll << z->slot_log2) < M) ++z->slot_log2;
    z->per_rank = cdiv(M, 1 << z->slot_log2);
    z->slots = z->per_rank * p->N;
    z->tiles_m = cdiv(z->slots, kBM >> z->slot_log2);
    const int want = cdiv(piece_rows ? piece_rows : kDefaultPiece, kBM);
    z->pieces = cdiv(z->tiles_m, want);
    z->piece_tiles = cdiv(z->tiles_m, z->pieces);
    z->pieces = cdiv(z->tiles_m, z->piece_tiles);
    z->tiles_v = cdiv(vocab, kBN);
    z->tiles_h = cdiv(hidden, kBN);
    z->pitch = (size_t)z->tiles_v * kBN;
    return BASP_OK;
}

struct Workspace {
    size_t cut, stats, scale, codes, info, kept, partial, acc, bytes;
};
Workspace workspace_of(const Sizes &z, int hidden, int vocab, bool grad) {
    Workspace w{};
    const size_t rows = (size_t)z.piece_tiles * kBM;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t o = at; at += up256(n); return o; };
    w.cut = take(rows * sizeof(float));
    w.stats = take(rows * z.tiles_v * (kBN / kStatCols) * sizeof(float2));
    if (grad) {
        w.scale = take(sizeof(unsigned));
        w.codes = take(rows * z.pitch * 2);
        w.info = take(rows * sizeof(RowInfo));
        w.kept = take(rows * hidden * 2);
        const int last = z.tiles_m - (z.pieces - 1) * z.piece_tiles, kb = cdiv(vocab, kBK);
        size_t partial = 0;                        // both sizes of piece, each with its own rows and splits
        for (int tiles : {z.piece_tiles, last}) {
            const int s = dx_splits(tiles, z.tiles_h, kb, hidden);
            const size_t bytes = s > 1 ? (size_t)s * tiles * kBM * hidden * 4 : 0;
            if (bytes > partial) partial = bytes;
        }
        w.partial = take(partial);
        w.acc = take(z.pieces > 1 ? (size_t)vocab * hidden * 4 : 0);
    }
    w.bytes = at;
    return w;
}

// 8192 rows of 4096 features: 6.83 / 6.31 / 6.14 / 5.98 / 6.26 ms with 1 / 2 / 4 / 8 / 16 row tiles (4 MiB each) in a group
constexpr long long kGroupBytes = 34 << 20;
constexpr int kPairBlocks = 8;                     // 128 rows (2 blocks of K): 609 us with single CTAs, 673 with pairs; 512 rows: alike

template <int kKind, int R, bool kPair>
int launch_as(const LossParams<R> &prm, cudaStream_t st) {
    const int smem = kStages * kStageBytes + (kKind == kDw ? 8 * kStagingBytes : 0) + 1024;
    int dev = 0;
    BASP_CUDA_TRY(cudaGetDevice(&dev));
    static std::atomic<int> sm_count[kMaxDevices];         // 0: this kernel has not been set up on the device
    int sms = dev < kMaxDevices ? sm_count[dev].load(std::memory_order_acquire) : 0;
    if (sms == 0) {
        BASP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        BASP_CUDA_TRY(cudaFuncSetAttribute(lm_gemm_kernel<kKind, R, kPair>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (dev < kMaxDevices) sm_count[dev].store(sms, std::memory_order_release);
    }
    const long long items = (long long)prm.tiles_m * prm.tiles_n * prm.splits, slots = kPair ? sms / 2 : sms;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(items < slots ? items : slots) * (kPair ? 2 : 1));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = kPair ? 2 : 1; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;         // (1) starts under lm_rows_kernel
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = kKind == kStats || kKind == kLogits ? 2 : 1;
    BASP_CUDA_TRY(cudaLaunchKernelEx(&cfg, lm_gemm_kernel<kKind, R, kPair>, prm));
    basp_count_launch(1);
    return BASP_OK;
}

// `rows`: of the product's first operand
template <int kKind, int R>
int launch_gemm(LossParams<R> &prm, int rows, cudaStream_t st) {
    // dW of few rows is all epilogue, and only single CTAs' tiles run one under the next tile's loads
    const bool pair = use_pair(rows) && !(kKind == kDw && prm.k_blocks < kPairBlocks);
    prm.tiles_m = cdiv(rows, pair ? kTileM<true> : kTileM<false>);
    // (1): as many row tiles as leave their x in L2 while W streams by; (2), (3): one, its dz streams once
    const long long tile_bytes = (long long)(pair ? kTileM<true> : kTileM<false>) * prm.hidden * 2;
    prm.group = kKind == kStats || kKind == kLogits ? (int)(kGroupBytes / tile_bytes) : 1;
    prm.group = prm.group < 1 ? 1 : (prm.group > prm.tiles_m ? prm.tiles_m : prm.group);
    return pair ? launch_as<kKind, R, true>(prm, st) : launch_as<kKind, R, false>(prm, st);
}

struct Args {
    int hidden, vocab;
    const void *const *x;
    const void *w;
    const long long *const *labels;
    const float *const *weights;
    float *const *loss, *const *lse;
    void *const *dx;
    void *dw;
    char *ws;
};

template <int R>
int run(const basp_plan *p, const Args &a, const Sizes &z, const Workspace &w, bool grad, cudaStream_t st) {
    const int M = p->Bl * p->T, M_last = p->Bl * p->T_last;
    const int slot = 1 << z.slot_log2, rows = z.piece_tiles * kBM;
    LossParams<R> prm;
    MergeParams<R> merge;
    memset(&prm, 0, sizeof(prm));
    memset(&merge, 0, sizeof(merge));
    prm.status = basp_status_device_ptr();
    if (!prm.status) return BASP_ERR_CUDA;
    prm.rows.slot_log2 = z.slot_log2; prm.rows.per_rank = z.per_rank; prm.rows.K = p->K; prm.rows.M = M; prm.rows.M_last = M_last;
    prm.vocab = a.vocab; prm.hidden = a.hidden; prm.pitch = z.pitch; prm.piece_rows = rows;
    prm.cut = (const float *)(a.ws + w.cut); prm.stats = (float2 *)(a.ws + w.stats); prm.scale = (unsigned *)(a.ws + w.scale);
    prm.codes = (uint16_t *)(a.ws + w.codes); prm.partial = (float *)(a.ws + w.partial);
    for (int r = 0; r < p->N; ++r) {
        prm.label[r] = a.labels[r];
        prm.dx[r] = a.dx ? (__nv_bfloat16 *)a.dx[r] : nullptr;
        merge.label[r] = a.labels[r];
        merge.x[r] = (const __nv_bfloat16 *)a.x[r];
        merge.weight[r] = a.weights ? a.weights[r] : nullptr;
        merge.loss[r] = a.loss[r];
        merge.lse[r] = a.lse ? a.lse[r] : nullptr;
    }
    merge.groups = z.tiles_v * (kBN / kStatCols); merge.piece_rows = rows; merge.vocab = a.vocab;
    merge.stats = prm.stats; merge.cut = prm.cut; merge.scale = prm.scale; merge.hidden = a.hidden; merge.w = (const __nv_bfloat16 *)a.w;
    merge.info = grad ? (RowInfo *)(a.ws + w.info) : nullptr;
    CUtensorMap w_k[2], w_mn, dz_k, dz_mn;     // w_k: of a single CTA, of a pair's
    for (int r = 0; r < p->N; ++r) {
        const uint64_t n = (uint64_t)p->Bl * basp_rank_tokens(p, r % p->K);
        BASP_TRY(tmap::encode_rows_heads_d(&prm.x[r], a.x[r], n, 1, a.hidden, slot));
    }
    for (int pair = 0; pair < 2; ++pair) BASP_TRY(tmap::encode_rows_heads_d(&w_k[pair], a.w, a.vocab, 1, a.hidden, kBN >> pair));
    if (grad) {
        BASP_TRY(tmap::encode_rows_heads_d(&w_mn, a.w, a.vocab, 1, a.hidden, kBK));
        BASP_TRY(tmap::encode_rows_heads_d(&dz_k, prm.codes, rows, 1, z.pitch, kBM));
        BASP_TRY(tmap::encode_rows_heads_d(&dz_mn, prm.codes, rows, 1, z.pitch, kBK));
        if (a.dw) BASP_TRY(tmap::encode_rows_heads_d(&prm.dw, a.dw, a.vocab, 1, a.hidden, 32));
        BASP_TRY(tmap::encode_rows_heads_d(&prm.kept, a.ws + w.kept, rows, 1, a.hidden, kBK));
    }
    CutParams<R> cut;
    memset(&cut, 0, sizeof(cut));
    for (int r = 0; r < p->N; ++r) cut.x[r] = (const __nv_bfloat16 *)a.x[r];
    cut.hidden = a.hidden; cut.cut = (float *)(a.ws + w.cut);
    bool wide_dx = a.hidden % 16 == 0;
    for (int r = 0; a.dx && r < p->N; ++r) wide_dx = wide_dx && (uintptr_t)a.dx[r] % 32 == 0;
    DzParams<R> dz;
    memset(&dz, 0, sizeof(dz));
    for (int r = 0; r < p->N; ++r) dz.x[r] = (const __nv_bfloat16 *)a.x[r];
    dz.kept = (__nv_bfloat16 *)(a.ws + w.kept); dz.codes = prm.codes; dz.pitch = z.pitch; dz.info = merge.info; dz.stats = prm.stats; dz.scale = prm.scale;
    dz.tiles_n = z.tiles_v; dz.piece_rows = rows; dz.hidden = a.hidden; dz.blocks = cdiv(z.tiles_v, 8 * kDzTiles);
    for (int piece = 0; piece < z.pieces; ++piece) {
        const int tile0 = piece * z.piece_tiles, tiles = tile0 + z.piece_tiles < z.tiles_m ? z.piece_tiles : z.tiles_m - tile0;
        const int per_tile = kBM >> z.slot_log2;
        prm.rows.slot_begin = tile0 * per_tile;
        prm.rows.slots = z.slots - prm.rows.slot_begin < tiles * per_tile ? z.slots - prm.rows.slot_begin : tiles * per_tile;
        merge.rows = prm.rows; cut.rows = prm.rows;
        lm_rows_kernel<R><<<tiles * kBM / 8, 256, 0, st>>>(cut);
        BASP_CUDA_TRY(cudaGetLastError());
        basp_count_launch(1);
        // (1)
        prm.tiles_n = z.tiles_v; prm.splits = 1; prm.k_blocks = cdiv(a.hidden, kBK);
        prm.w = w_k[use_pair(tiles * kBM)];
        if (grad) BASP_TRY((launch_gemm<kLogits, R>(prm, tiles * kBM, st)));
        else BASP_TRY((launch_gemm<kStats, R>(prm, tiles * kBM, st)));
        BASP_CUDA_TRY(launch_early(lm_merge_kernel<R>, dim3(tiles * kBM / 32), 1024, st, merge));
        basp_count_launch(1);
        if (!grad) continue;
        dz.rows = prm.rows;
        lm_dz_kernel<R><<<dim3(dz.blocks + (a.dw ? 1 : 0), tiles * kBM), 256, 0, st>>>(dz);
        BASP_CUDA_TRY(cudaGetLastError());
        basp_count_launch(1);
        // (2)
        if (a.dx) {
            prm.w = w_mn;
            prm.dz = dz_k;
            prm.tiles_n = z.tiles_h; prm.k_blocks = cdiv(a.vocab, kBK); prm.wide = wide_dx;
            prm.splits = dx_splits(tiles, z.tiles_h, prm.k_blocks, a.hidden);
            prm.partial_rows = tiles * kBM;
            BASP_TRY((launch_gemm<kDx, R>(prm, tiles * kBM, st)));
            if (prm.splits > 1) {
                JoinParams<R> join;
                memcpy(join.dx, prm.dx, sizeof(join.dx));
                join.rows = prm.rows; join.partial = prm.partial; join.splits = prm.splits; join.partial_rows = prm.partial_rows; join.hidden = a.hidden;
                BASP_CUDA_TRY(launch_early(lm_dx_join_kernel<R>, dim3(cdiv((long long)tiles * kBM * (a.hidden / 8), 256)), 256, st, join));
                basp_count_launch(1);
            }
        }
        // (3)
        if (a.dw) {
            prm.dz = dz_mn;
            prm.tiles_n = z.tiles_h; prm.splits = 1;
            prm.k_blocks = cdiv((long long)prm.rows.slots << z.slot_log2, kBK);
            prm.acc_in = piece > 0 ? (const float *)(a.ws + w.acc) : nullptr;
            prm.acc_out = piece + 1 < z.pieces ? (float *)(a.ws + w.acc) : nullptr;
            BASP_TRY((launch_gemm<kDw, R>(prm, a.vocab, st)));
        }
    }
    return BASP_OK;
}

int call(const basp_plan *p, const Args &a, bool grad, int piece_rows, size_t workspace_bytes, void *stream) {
    if (!p) return BASP_ERR_NULL;
    Sizes z;
    BASP_TRY(sizes_of(p, a.hidden, a.vocab, piece_rows, &z));
    const Workspace w = workspace_of(z, a.hidden, a.vocab, grad);
    SpanSet spans;
    if (!a.x || !a.labels || !a.loss || (grad && !a.dx && !a.dw)) return BASP_ERR_NULL;
    const size_t w_bytes = (size_t)a.vocab * a.hidden * 2;
    BASP_TRY(spans.add_in(a.w, w_bytes));
    for (int r = 0; r < p->N; ++r) {
        const size_t n = (size_t)p->Bl * basp_rank_tokens(p, r % p->K);
        BASP_TRY(spans.add_in(a.x[r], n * a.hidden * 2));
        BASP_TRY(spans.add_in(a.labels[r], n * 8, 8));
        if (a.weights) BASP_TRY(spans.add_in(a.weights[r], n * 4, 4));
        BASP_TRY(spans.add_out(a.loss[r], n * 4, 4));
        if (a.lse) BASP_TRY(spans.add_out(a.lse[r], n * 4, 4));
        if (a.dx) BASP_TRY(spans.add_out(a.dx[r], n * a.hidden * 2));
    }
    if (a.dw) BASP_TRY(spans.add_out(a.dw, w_bytes));
    BASP_TRY(spans.add_out(a.ws, w.bytes));
    if (workspace_bytes < w.bytes) return BASP_ERR_WORKSPACE;
    BASP_TRY(spans.overlaps());
    if (p->N <= 8) return run<8>(p, a, z, w, grad, (cudaStream_t)stream);
    return run<BASP_MAX_RANKS>(p, a, z, w, grad, (cudaStream_t)stream);
}

}  // namespace

extern "C" size_t basp_lm_loss_fwd_workspace_bytes(const basp_plan *p, int vocab) {
    Sizes z;
    if (!p || sizes_of(p, 8, vocab, 0, &z) != BASP_OK) return 0;
    return workspace_of(z, 8, vocab, false).bytes;
}

extern "C" int basp_lm_loss_fwd(const basp_plan *p, int hidden, int vocab, const void *const *x_seq, const void *w,
                                const long long *const *labels, float *const *loss_seq, float *const *lse_seq, void *workspace,
                                size_t workspace_bytes, void *stream) {
    const Args a{hidden, vocab, x_seq, w, labels, nullptr, loss_seq, lse_seq, nullptr, nullptr, (char *)workspace};
    return call(p, a, false, 0, workspace_bytes, stream);
}

extern "C" size_t basp_lm_loss_grad_workspace_bytes(const basp_plan *p, int hidden, int vocab, int piece_rows) {
    Sizes z;
    if (!p || sizes_of(p, hidden, vocab, piece_rows, &z) != BASP_OK) return 0;
    return workspace_of(z, hidden, vocab, true).bytes;
}

extern "C" int basp_lm_loss_grad(const basp_plan *p, int hidden, int vocab, const void *const *x_seq, const void *w,
                                 const long long *const *labels, const float *const *token_weights, float *const *loss_seq,
                                 float *const *lse_seq, void *const *dx_seq, void *dw, int piece_rows, void *workspace,
                                 size_t workspace_bytes, void *stream) {
    const Args a{hidden, vocab, x_seq, w, labels, token_weights, loss_seq, lse_seq, dx_seq, dw, (char *)workspace};
    return call(p, a, true, piece_rows, workspace_bytes, stream);
}
