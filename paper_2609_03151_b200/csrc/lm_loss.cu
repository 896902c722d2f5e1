// Softmax cross entropy of the language-model head over a large vocabulary, on all ranks' sequence shards, without keeping
// the logits; alone, and with its gradients.  For a token with hidden state x, label y and weight g:
//
//   z = x W^T,   lse = ln sum_v exp z_v,   loss = lse - z_y,
//   dz = g (softmax(z) - onehot(y)),       dx = dz W,       dW = sum_tokens dz^T x
//
// Three products, each 2 rows*vocab*hidden operations on the tensor cores, and one element-wise pass:
//   (1) z = x W^T          epilogue: per row and 256-column tile the maximum m and the sum of exp(z - m), the target's
//                          logit apart from the others; for the gradient also every logit as its distance below the tile's
//                          maximum, 16 bits: rn((m - z) log2(e) 2^10), saturating at 2^-64 of the maximum's probability
//   (merge)                rows' statistics -> loss and lse
//   (dz)                   in place: 16-bit distance -> bf16 dz (and the piece's rows of x side by side for (3), those without a
//                          part in the gradients as zeros: 0 x NaN would reach every word's gradient).  A distance is off by at most 2^-11 in log2, so the
//                          probability by 2^-11 ln 2 = 3.4e-4, against bf16's own 2^-8: the 16 bits cost a fifth of nothing
//                          and save half of an fp32 logit's traffic and memory
//   (2) dx = dz W          split over the vocabulary where there are too few row tiles for all SMs (fp32 partial sums, joined
//                          by one more pass)
//   (3) dW = dz^T x        K = the piece's rows; with several pieces the sum is carried in fp32
// The rows are worked on in pieces (default 8192), so the memory between the products is 2 bytes per logit of one piece.
//
// The target's logit is left out of the sums: with o = ln sum_{v != y} exp z_v, loss = softplus(o - z_y) and the target's
// dz = -g sigmoid(o - z_y).  lse - z_y and p_y - 1 would cancel for a confident prediction.
//
// Products: persistent, one CTA per SM, tile 128 x 256, K in blocks of 64 (128-byte-swizzled TMA boxes):
//   warp 0      TMA producer, 4-stage ring (A 16 KiB + B 32 KiB per stage)
//   warp 1      tcgen05.mma issuer (M = 128, N = 256, K = 16), two 256-column TMEM accumulators so that the epilogue of one
//               tile runs under the main loop of the next
//   warps 2-5   epilogue (a thread owns a row of the tile)
// W and x are read as they lie: K-major for (1), and as MN-major operands for (2) and (3), dz K-major for (2) and MN-major for
// (3); nothing is transposed in memory.
//
// Rows of all ranks are put together in slots of 8..128 rows (a power of two, by the rows of a rank), so that a tile holds
// several ranks where a rank has few tokens; rows of a slot past a rank's end are zero in every product.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include "common.cuh"
#include "ptx.cuh"
#include "spans.h"
#include "tmap.cuh"

int *basp_status_device_ptr();

namespace {

using namespace ptx;

constexpr int kThreads = 192;
constexpr int kBM = 128, kBN = 256, kBK = 64, kStages = 4;
constexpr int kABytes = kBM * kBK * 2, kBBytes = kBN * kBK * 2;
constexpr int kMnBlock = kBK * 64 * 2;             // one 64-column block of an MN-major operand: 64 rows of 128 bytes
constexpr int kSms = 148;                          // of the GPU this code is written for; plans the split, not the grid
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
    CUtensorMap x[R];          // (1): boxes of a slot's rows
    CUtensorMap w, dz;
    CUtensorMap kept;          // (3): the piece's rows of x, zero where a row has no part in the gradients
    const long long *label[R];
    __nv_bfloat16 *dx[R];
    Rows rows;
    int tiles_m, tiles_n, k_blocks, splits;
    int vocab, hidden;
    size_t pitch;              // columns of a row of 16-bit logits
    int piece_rows;
    float2 *stats;             // [tiles_n][piece_rows]: maximum, sum
    float *target;             // [piece_rows]: the target's logit
    uint16_t *codes;           // [piece_rows][pitch]
    float *partial;            // (2) with splits > 1: [splits][piece_rows][hidden]
    const float *acc_in;       // (3) sum of the earlier pieces, or NULL
    float *acc_out;            // (3) sum so far, or NULL: the result
    __nv_bfloat16 *dw;
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

// Tile coordinates of a work item.  (1): row tiles fastest, so the piece's x stays in L2 and W streams once; (2), (3):
// column tiles of `hidden` fastest.
struct Item {
    int m, n, kb0, kb1, split;
};
template <int kKind, int R>
__device__ __forceinline__ Item item_of(const LossParams<R> &p, int i) {
    Item t;
    t.split = 0; t.kb0 = 0; t.kb1 = p.k_blocks;
    if constexpr (kKind == kStats || kKind == kLogits) {
        t.n = i / p.tiles_m;
        t.m = i - t.n * p.tiles_m;
    } else {
        const int q = i / p.tiles_n;
        t.n = i - q * p.tiles_n;
        t.split = kKind == kDx ? q / p.tiles_m : 0;
        t.m = q - t.split * p.tiles_m;
        if constexpr (kKind == kDx) {
            t.kb0 = (int)((long long)p.k_blocks * t.split / p.splits);
            t.kb1 = (int)((long long)p.k_blocks * (t.split + 1) / p.splits);
        }
    }
    return t;
}

__device__ __forceinline__ void store_bf16x32(__nv_bfloat16 *dst, const float (&v)[32], int cols) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (8 * i >= cols) break;                  // cols is a multiple of 8
        uint4 o;
        o.x = pack_bf16x2(v[8 * i + 0], v[8 * i + 1]); o.y = pack_bf16x2(v[8 * i + 2], v[8 * i + 3]);
        o.z = pack_bf16x2(v[8 * i + 4], v[8 * i + 5]); o.w = pack_bf16x2(v[8 * i + 6], v[8 * i + 7]);
        *reinterpret_cast<uint4 *>(dst + 8 * i) = o;
    }
}

template <int kKind, int R>
__global__ void __launch_bounds__(kThreads, 1) lm_gemm_kernel(const __grid_constant__ LossParams<R> p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sA = smem;                                    // kStages x 16 KiB
    uint8_t *sB = smem + kStages * kABytes;                // kStages x 32 KiB
    __shared__ Bars bars;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int total = p.tiles_m * p.tiles_n * p.splits;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&bars.full[s], 1); mbar_init(&bars.empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&bars.acc_full[a], 1); mbar_init(&bars.acc_empty[a], 4); }
        bars.abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) { tmem_alloc(&bars.tmem_base, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars.tmem_base;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer (lane 0 issues)
        uint32_t it = 0;
        for (int i = blockIdx.x; i < total; i += gridDim.x) {
            const Item t = item_of<kKind>(p, i);
            for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
                const uint32_t s = it % kStages, ph = (it / kStages) & 1;
                LOSS_WAIT(&bars.empty[s], ph ^ 1, 0, kb);
                if (lane == 0) {
                    uint8_t *a = sA + s * kABytes, *b = sB + s * kBBytes;
                    mbar_arrive_expect_tx(&bars.full[s], kABytes + kBBytes);
                    if constexpr (kKind == kStats || kKind == kLogits) {
                        // a slot past the piece's end is read past its rank's last row: zeros
                        const int slot = 1 << p.rows.slot_log2;
                        for (int j = 0; j < kBM; j += slot) {
                            const int sl = (t.m * kBM + j) >> p.rows.slot_log2, at = p.rows.slot_begin + sl;
                            const bool in = sl < p.rows.slots;
                            const int r = in ? at / p.rows.per_rank : 0;
                            tma_load_3d(a + j * kBK * 2, &p.x[r], &bars.full[s], kb * kBK, 0,
                                        (in ? at - r * p.rows.per_rank : p.rows.per_rank) << p.rows.slot_log2);
                        }
                        tma_load_3d(b, &p.w, &bars.full[s], kb * kBK, 0, t.n * kBN);
                    } else if constexpr (kKind == kDx) {
                        tma_load_3d(a, &p.dz, &bars.full[s], kb * kBK, 0, t.m * kBM);
#pragma unroll
                        for (int c = 0; c < kBN / 64; ++c)
                            tma_load_3d(b + c * kMnBlock, &p.w, &bars.full[s], t.n * kBN + c * 64, 0, kb * kBK);
                    } else {
#pragma unroll
                        for (int c = 0; c < kBM / 64; ++c)
                            tma_load_3d(a + c * kMnBlock, &p.dz, &bars.full[s], t.m * kBM + c * 64, 0, kb * kBK);
#pragma unroll
                        for (int c = 0; c < kBN / 64; ++c)
                            tma_load_3d(b + c * kMnBlock, &p.kept, &bars.full[s], t.n * kBN + c * 64, 0, kb * kBK);
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (lane 0 issues)
        const uint32_t idesc = make_idesc_bf16(kBM, kBN, kKind == kDw, kKind == kDx || kKind == kDw);
        const uint64_t desc_k = make_smem_desc_sw128(0, 16, 1024), desc_mn = make_smem_desc_sw128(0, kMnBlock, 1024);
        const uint64_t da0 = (kKind == kDw ? desc_mn : desc_k) | (uint64_t)(smem_u32(sA) >> 4);
        const uint64_t db0 = (kKind == kDx || kKind == kDw ? desc_mn : desc_k) | (uint64_t)(smem_u32(sB) >> 4);
        // 16 elements of K: 32 bytes along a row, or 16 rows of 128 bytes
        constexpr int kStepA = kKind == kDw ? 128 : 2, kStepB = kKind == kDx || kKind == kDw ? 128 : 2;
        uint32_t it = 0, cnt = 0;
        for (int i = blockIdx.x; i < total; i += gridDim.x, ++cnt) {
            const Item t = item_of<kKind>(p, i);
            const uint32_t acc = cnt & 1;
            LOSS_WAIT(&bars.acc_empty[acc], ((cnt >> 1) & 1) ^ 1, 1, i);
            tc_fence_after();
            for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
                const uint32_t s = it % kStages, ph = (it / kStages) & 1;
                LOSS_WAIT(&bars.full[s], ph, 2, kb);
                tc_fence_after();
                if (lane == 0) {
                    const uint64_t da = da0 + s * (kABytes >> 4), db = db0 + s * (kBBytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < kBK / 16; ++kk)
                        mma_ss(tmem + acc * kBN, da + kk * kStepA, db + kk * kStepB, idesc, (kb > t.kb0) || (kk > 0));
                    tc_commit(&bars.empty[s]);
                }
            }
            if (lane == 0) tc_commit(&bars.acc_full[acc]);
        }
    } else {
        // ------------------------------------------------------------------ epilogue (warps 2..5)
        const int quarter = warp & 3;                       // the TMEM lanes this warp can reach
        const int row = quarter * 32 + lane;
        const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
        uint32_t cnt = 0;
        for (int i = blockIdx.x; i < total; i += gridDim.x, ++cnt) {
            const Item t = item_of<kKind>(p, i);
            const uint32_t acc = cnt & 1;
            const uint32_t src = tmem + acc * kBN + lane_addr;
            const int prow = t.m * kBM + row;
            const int col0 = t.n * kBN;
            if constexpr (kKind == kStats || kKind == kLogits) {
                const Token tok = token_of(p.rows, prow);
                const long long label = tok.valid ? p.label[tok.rank][tok.row] : -1;
                // the target's column in this tile, or -1
                const int hit = label >= col0 && label < p.vocab && label < col0 + kBN ? (int)(label - col0) : -1;
                const int cols = min(kBN, p.vocab - col0);
                LOSS_WAIT(&bars.acc_full[acc], (cnt >> 1) & 1, 3, i);
                tc_fence_after();
                float m = -INFINITY;
                for (int c = 0; c < kBN / 32; ++c) {
                    uint32_t v[32];
                    tmem_ld_x32(src + c * 32, v);
                    tmem_wait_ld();
                    const bool special = __any_sync(0xffffffffu, (hit >> 5) == c) || cols < c * 32 + 32;
                    if (!special) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) m = max3(m, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const float z = __uint_as_float(v[e]);
                            if (c * 32 + e == hit) p.target[prow] = z;
                            else if (c * 32 + e < cols) m = fmaxf(m, z);
                        }
                    }
                }
                const float top = m == -INFINITY ? 0.f : m;         // nothing but the target: distances are infinite
                float sum = 0.f;
                uint16_t *dst = p.codes + (size_t)prow * p.pitch + col0;
                for (int c = 0; c < kBN / 32; ++c) {
                    uint32_t v[32];
                    tmem_ld_x32(src + c * 32, v);
                    tmem_wait_ld();
                    if (c == kBN / 32 - 1) {                        // the accumulator is in registers: hand it back
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars.acc_empty[acc]);
                    }
                    const bool special = __any_sync(0xffffffffu, (hit >> 5) == c) || cols < c * 32 + 32;
                    uint32_t out[16];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float d = (top - __uint_as_float(v[e])) * kLog2e;
                        if (special && (c * 32 + e == hit || c * 32 + e >= cols)) d = INFINITY;
                        sum += exp2_approx(-d);
                        if constexpr (kKind == kLogits) {
                            // + 2^23: the nearest whole number in the low bits
                            const uint32_t code = __float_as_uint(fminf(d * kCodeStep, kCodeMax) + 8388608.f);
                            if (e & 1) out[e / 2] = __byte_perm(out[e / 2], code, 0x5410);
                            else out[e / 2] = code;
                        }
                    }
                    if constexpr (kKind == kLogits) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            *reinterpret_cast<uint4 *>(dst + c * 32 + 8 * q) = make_uint4(out[4 * q], out[4 * q + 1], out[4 * q + 2], out[4 * q + 3]);
                    }
                }
                p.stats[(size_t)t.n * p.piece_rows + prow] = make_float2(m, sum);
            } else {
                const int width = min(kBN, p.hidden - col0);        // a multiple of 8
                Token tok{0, prow, prow < p.vocab};
                if constexpr (kKind == kDx) tok = token_of(p.rows, prow);
                LOSS_WAIT(&bars.acc_full[acc], (cnt >> 1) & 1, 3, i);
                tc_fence_after();
                for (int c = 0; c < kBN / 32; ++c) {
                    uint32_t raw[32];
                    tmem_ld_x32(src + c * 32, raw);
                    tmem_wait_ld();
                    if (c == kBN / 32 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars.acc_empty[acc]);
                    }
                    const int cols = min(32, width - c * 32);
                    if (!tok.valid || cols <= 0) continue;
                    float v[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(raw[e]);
                    if constexpr (kKind == kDx) {
                        if (p.splits == 1) {
                            store_bf16x32(p.dx[tok.rank] + (size_t)tok.row * p.hidden + col0 + c * 32, v, cols);
                        } else {
                            float *dst = p.partial + ((size_t)t.split * p.piece_rows + prow) * p.hidden + col0 + c * 32;
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                if (4 * q < cols) *reinterpret_cast<float4 *>(dst + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                        }
                    } else {
                        const size_t at = (size_t)prow * p.hidden + col0 + c * 32;
                        if (p.acc_in) {
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                if (4 * q < cols) {
                                    const float4 o = *reinterpret_cast<const float4 *>(p.acc_in + at + 4 * q);
                                    v[4 * q] += o.x; v[4 * q + 1] += o.y; v[4 * q + 2] += o.z; v[4 * q + 3] += o.w;
                                }
                        }
                        if (p.acc_out) {
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                if (4 * q < cols) *reinterpret_cast<float4 *>(p.acc_out + at + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                        } else {
                            store_bf16x32(p.dw + at, v, cols);
                        }
                    }
                }
            }
        }
    }

gemm_done:
    tc_fence_before();
    __syncthreads();
    if (bars.abort_flag) {
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) { }
        __syncthreads();
    }
    if (warp == 1) tmem_dealloc(tmem, 512);
}

#undef LOSS_WAIT

// ------------------------------------------------------------------------------------------------ statistics of the rows
struct RowInfo {               // what the element-wise pass needs of a row
    float lse, weight, target_dz;
    int label;                 // -1: none
};

template <int R>
struct MergeParams {
    const long long *label[R];
    const float *weight[R];    // a NULL table entry: weight 1
    float *loss[R], *lse[R];
    Rows rows;
    int tiles_n, piece_rows, vocab;
    const float2 *stats;
    const float *target;
    RowInfo *info;             // NULL: not wanted
};

__device__ __forceinline__ void join(float &m, float &s, float m2, float s2) {
    const float top = fmaxf(m, m2), use = top == -INFINITY ? 0.f : top;
    s = s * exp2f((m - use) * kLog2e) + s2 * exp2f((m2 - use) * kLog2e);
    m = top;
}

// A block takes 32 rows; its 32 warps share the tiles of a row (neighbouring lanes read neighbouring rows).
template <int R>
__global__ void __launch_bounds__(1024) lm_merge_kernel(const __grid_constant__ MergeParams<R> p) {
    __shared__ float2 part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    float m = -INFINITY, s = 0.f;
    constexpr int kBatch = 8;                      // loads in flight
    for (int n0 = warp; n0 < p.tiles_n; n0 += 32 * kBatch) {
        float2 v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int n = n0 + 32 * u;
            v[u] = n < p.tiles_n ? p.stats[(size_t)n * p.piece_rows + i] : make_float2(-INFINITY, 0.f);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) join(m, s, v[u].x, v[u].y);
    }
    part[warp][lane] = make_float2(m, s);
    __syncthreads();
    if (warp != 0) return;
    for (int w = 1; w < 32; ++w) join(m, s, part[w][lane].x, part[w][lane].y);
    const Token tok = token_of(p.rows, i);
    RowInfo info{0.f, 0.f, 0.f, -1};
    if (tok.valid) {
        const float others = m + logf(s);          // -inf where the target is the only word
        const long long label = p.label[tok.rank][tok.row];
        float loss = 0.f, lse = others;
        if (label >= 0 && label < p.vocab) {
            const float z = p.target[i], away = others - z, tail = log1pf(expf(-fabsf(away)));
            loss = (away > 0.f ? away : 0.f) + tail;
            lse = (away > 0.f ? others : z) + tail;
            if (p.info) {
                const float g = p.weight[tok.rank] ? p.weight[tok.rank][tok.row] : 1.f;
                info.weight = g;
                info.target_dz = -g / (1.f + expf(-away));
                info.label = (int)label;
            }
        }
        info.lse = lse;
        p.loss[tok.rank][tok.row] = loss;
        if (p.lse[tok.rank]) p.lse[tok.rank][tok.row] = lse;
    }
    if (p.info) p.info[i] = info;
}

// ------------------------------------------------------------------------------------------------ 16-bit distances -> bf16 dz
// In place.  A warp takes 256-column tiles of one row (the tile's maximum is one value for the warp), a lane 8 columns.  A row
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
    const int n0 = (blockIdx.x * 8 + warp) * kDzTiles;
    uint4 v[kDzTiles];
    float m[kDzTiles];
    uint4 *at = reinterpret_cast<uint4 *>(p.codes + (size_t)row * p.pitch) + (size_t)n0 * 32 + lane;
    if (info.weight != 0.f) {
#pragma unroll
        for (int u = 0; u < kDzTiles; ++u)
            if (n0 + u < tiles_n) {
                v[u] = at[u * 32];
                m[u] = __ldg(&p.stats[(size_t)(n0 + u) * piece_rows + row].x);
            }
    }
#pragma unroll
    for (int u = 0; u < kDzTiles; ++u) {
        if (n0 + u >= tiles_n) break;
        uint4 o = make_uint4(0, 0, 0, 0);
        if (info.weight != 0.f) {
            const float c = (m[u] - info.lse) * kLog2e;
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
                    d[e] = 2 * q + e == target ? info.target_dz : exp2_approx(c - dist) * info.weight;
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
    int splits, piece_rows, hidden;
};
template <int R>
__global__ void __launch_bounds__(256) lm_dx_join_kernel(const __grid_constant__ JoinParams<R> p) {
    const int per_row = p.hidden / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(i / per_row), c = (int)(i - (long long)row * per_row) * 8;
    if (row >= p.piece_rows) return;
    const Token tok = token_of(p.rows, row);
    if (!tok.valid) return;
    float s[8] = {};
    for (int k = 0; k < p.splits; ++k) {
        const float4 *src = reinterpret_cast<const float4 *>(p.partial + ((size_t)k * p.piece_rows + row) * p.hidden + c);
        const float4 a = src[0], b = src[1];
        s[0] += a.x; s[1] += a.y; s[2] += a.z; s[3] += a.w; s[4] += b.x; s[5] += b.y; s[6] += b.z; s[7] += b.w;
    }
    uint4 o;
    o.x = pack_bf16x2(s[0], s[1]); o.y = pack_bf16x2(s[2], s[3]); o.z = pack_bf16x2(s[4], s[5]); o.w = pack_bf16x2(s[6], s[7]);
    *reinterpret_cast<uint4 *>(p.dx[tok.rank] + (size_t)tok.row * p.hidden + c) = o;
}

// ------------------------------------------------------------------------------------------------ host side
constexpr int kDefaultPiece = 8192, kMaxPiece = 32768;
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
int cdiv(long long a, long long b) { return (int)((a + b - 1) / b); }

// Sizes of one call: slots, pieces, and the workspace.
struct Sizes {
    int slot_log2, per_rank, slots;                // slots of all ranks
    int tiles_m, piece_tiles, pieces;              // row tiles in all and per piece
    int tiles_v, tiles_h;                          // 256-column tiles of the vocabulary and of `hidden`
    size_t pitch;
};

// How often the vocabulary is split in dx = dz W: the time of `waves` rounds of tiles over the SMs, a tile costing its K
// blocks plus a start and an epilogue (8 blocks), plus writing and reading the partial sums.
int dx_splits(int tiles_m, int tiles_h, int k_blocks, int hidden) {
    const double block_us = 0.43;                  // 128 x 256 x 64 at the sustained rate of one SM
    int best = 1;
    double best_us = 1e30;
    for (int s = 1; s <= 64 && (s == 1 || k_blocks / s >= 8); ++s) {
        const double bytes = (double)s * tiles_m * kBM * hidden * 4;
        if (s > 1 && bytes > 256e6) break;
        const double us = (double)cdiv((long long)tiles_m * tiles_h * s, kSms) * (cdiv(k_blocks, s) + 8) * block_us +
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
    size_t stats, target, codes, info, kept, partial, acc, bytes;
};
Workspace workspace_of(const Sizes &z, int hidden, int vocab, bool grad) {
    Workspace w{};
    const size_t rows = (size_t)z.piece_tiles * kBM;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t o = at; at += up256(n); return o; };
    w.stats = take(rows * z.tiles_v * sizeof(float2));
    w.target = take(rows * sizeof(float));
    if (grad) {
        w.codes = take(rows * z.pitch * 2);
        w.info = take(rows * sizeof(RowInfo));
        w.kept = take(rows * hidden * 2);
        const int last = z.tiles_m - (z.pieces - 1) * z.piece_tiles, kb = cdiv(vocab, kBK);
        size_t partial = 0;
        for (int tiles : {z.piece_tiles, last}) {
            const int s = dx_splits(tiles, z.tiles_h, kb, hidden);
            if (s > 1 && (size_t)s * tiles * kBM * hidden * 4 > partial) partial = (size_t)s * tiles * kBM * hidden * 4;
        }
        w.partial = take(partial);
        w.acc = take(z.pieces > 1 ? (size_t)vocab * hidden * 4 : 0);
    }
    w.bytes = at;
    return w;
}

template <int kKind, int R>
int launch_gemm(const LossParams<R> &prm, cudaStream_t st) {
    int dev = 0, sms = 0;
    BASP_CUDA_TRY(cudaGetDevice(&dev));
    BASP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const long long items = (long long)prm.tiles_m * prm.tiles_n * prm.splits;
    const int smem = kStages * (kABytes + kBBytes) + 1024;
    BASP_CUDA_TRY(cudaFuncSetAttribute(lm_gemm_kernel<kKind, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    lm_gemm_kernel<kKind, R><<<(int)(items < sms ? items : sms), kThreads, smem, st>>>(prm);
    BASP_CUDA_TRY(cudaGetLastError());
    basp_count_launch(1);
    return BASP_OK;
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
    prm.stats = (float2 *)(a.ws + w.stats); prm.target = (float *)(a.ws + w.target);
    prm.codes = (uint16_t *)(a.ws + w.codes); prm.partial = (float *)(a.ws + w.partial);
    prm.dw = (__nv_bfloat16 *)a.dw;
    for (int r = 0; r < p->N; ++r) {
        prm.label[r] = a.labels[r];
        prm.dx[r] = a.dx ? (__nv_bfloat16 *)a.dx[r] : nullptr;
        merge.label[r] = a.labels[r];
        merge.weight[r] = a.weights ? a.weights[r] : nullptr;
        merge.loss[r] = a.loss[r];
        merge.lse[r] = a.lse ? a.lse[r] : nullptr;
    }
    merge.tiles_n = z.tiles_v; merge.piece_rows = rows; merge.vocab = a.vocab;
    merge.stats = prm.stats; merge.target = prm.target;
    merge.info = grad ? (RowInfo *)(a.ws + w.info) : nullptr;
    CUtensorMap w_k, w_mn, dz_k, dz_mn;
    for (int r = 0; r < p->N; ++r) {
        const uint64_t n = (uint64_t)p->Bl * basp_rank_tokens(p, r % p->K);
        BASP_TRY(tmap::encode_rows_heads_d(&prm.x[r], a.x[r], n, 1, a.hidden, slot));
    }
    BASP_TRY(tmap::encode_rows_heads_d(&w_k, a.w, a.vocab, 1, a.hidden, kBN));
    if (grad) {
        BASP_TRY(tmap::encode_rows_heads_d(&w_mn, a.w, a.vocab, 1, a.hidden, kBK));
        BASP_TRY(tmap::encode_rows_heads_d(&dz_k, prm.codes, rows, 1, z.pitch, kBM));
        BASP_TRY(tmap::encode_rows_heads_d(&dz_mn, prm.codes, rows, 1, z.pitch, kBK));
        BASP_TRY(tmap::encode_rows_heads_d(&prm.kept, a.ws + w.kept, rows, 1, a.hidden, kBK));
    }
    DzParams<R> dz;
    memset(&dz, 0, sizeof(dz));
    for (int r = 0; r < p->N; ++r) dz.x[r] = (const __nv_bfloat16 *)a.x[r];
    dz.kept = (__nv_bfloat16 *)(a.ws + w.kept); dz.codes = prm.codes; dz.pitch = z.pitch; dz.info = merge.info; dz.stats = prm.stats;
    dz.tiles_n = z.tiles_v; dz.piece_rows = rows; dz.hidden = a.hidden; dz.blocks = cdiv(z.tiles_v, 8 * kDzTiles);
    for (int piece = 0; piece < z.pieces; ++piece) {
        const int tile0 = piece * z.piece_tiles, tiles = tile0 + z.piece_tiles < z.tiles_m ? z.piece_tiles : z.tiles_m - tile0;
        const int per_tile = kBM >> z.slot_log2;
        prm.rows.slot_begin = tile0 * per_tile;
        prm.rows.slots = z.slots - prm.rows.slot_begin < tiles * per_tile ? z.slots - prm.rows.slot_begin : tiles * per_tile;
        merge.rows = prm.rows;
        // (1)
        prm.w = w_k;
        prm.tiles_m = tiles; prm.tiles_n = z.tiles_v; prm.splits = 1; prm.k_blocks = cdiv(a.hidden, kBK);
        if (grad) BASP_TRY((launch_gemm<kLogits, R>(prm, st)));
        else BASP_TRY((launch_gemm<kStats, R>(prm, st)));
        lm_merge_kernel<R><<<tiles * kBM / 32, 1024, 0, st>>>(merge);
        BASP_CUDA_TRY(cudaGetLastError());
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
            prm.tiles_n = z.tiles_h; prm.k_blocks = cdiv(a.vocab, kBK);
            prm.splits = dx_splits(tiles, z.tiles_h, prm.k_blocks, a.hidden);
            BASP_TRY((launch_gemm<kDx, R>(prm, st)));
            if (prm.splits > 1) {
                JoinParams<R> join;
                memcpy(join.dx, prm.dx, sizeof(join.dx));
                join.rows = prm.rows; join.partial = prm.partial; join.splits = prm.splits; join.piece_rows = rows; join.hidden = a.hidden;
                lm_dx_join_kernel<R><<<cdiv((long long)tiles * kBM * (a.hidden / 8), 256), 256, 0, st>>>(join);
                BASP_CUDA_TRY(cudaGetLastError());
                basp_count_launch(1);
            }
        }
        // (3)
        if (a.dw) {
            prm.dz = dz_mn;
            prm.tiles_m = cdiv(a.vocab, kBM); prm.tiles_n = z.tiles_h; prm.splits = 1;
            prm.k_blocks = cdiv((long long)prm.rows.slots << z.slot_log2, kBK);
            prm.acc_in = piece > 0 ? (const float *)(a.ws + w.acc) : nullptr;
            prm.acc_out = piece + 1 < z.pieces ? (float *)(a.ws + w.acc) : nullptr;
            BASP_TRY((launch_gemm<kDw, R>(prm, st)));
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
