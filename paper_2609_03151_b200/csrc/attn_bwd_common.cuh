// What the backward kernels of the attention share: warp roles, barriers, and the helper kernels around the products
// (Delta = rowsum(dO * O); the fp32 dQ accumulator to bf16).
#pragma once
#include <cuda_bf16.h>

#include "common.cuh"
#include "ptx.cuh"

namespace {

using namespace ptx;

constexpr int kT = 128;
constexpr int kBwdComputeWarps = 16;
[[maybe_unused]] constexpr int kBwdDrainWarp0 = kBwdComputeWarps;          // 4 warps that take dQ out of TMEM and reduce-add it
constexpr int kBwdTmaWarp = kBwdComputeWarps + 4;
constexpr int kBwdMmaWarp = kBwdComputeWarps + 5;
constexpr int kBwdThreads = (kBwdComputeWarps + 8) * 32;   // + drain warpgroup + (TMA, MMA, two idle warps)

struct BwdBars {
    uint64_t kv_full, kv_empty, qdo_full[3], qdo_empty[2], qdo_mma_done[3];      // (Q / dO stages: the 64-wide kernel has three)
    uint64_t s_full, stats_full[3], pds_ready, dq_full, dq_read, dkdv_full, dkdv_read;
    uint64_t s_full_b[2], dp_full, p_ready;   // the pipelined kernels: one S^T barrier per buffer, dP^T and P^T on their own
    uint64_t do_full[2], do_free[2];          // the pipelined 128-wide kernel: dO stages are released on their own
    uint32_t tmem_base;
    int abort_flag;
};

__device__ __forceinline__ void bwd_report(int *status, int code, int role, int detail) {
    if (atomicCAS(status, 0, code) == 0) {
        status[1] = role;
        status[2] = (int)blockIdx.x;
        status[3] = detail;
    }
}

#define BWD_WAIT(bar, parity, role, detail)                                    \
    do {                                                                        \
        if (!mbar_wait((bar), (parity), &bars->abort_flag)) {                  \
            bars->abort_flag = 1;                                               \
            bwd_report(p.status, 3, (role), (detail));                          \
            goto bwd_done;                                                      \
        }                                                                       \
    } while (0)

// Delta[bl][h][s] = sum_d O[bl][s][h][d] * dO[bl][s][h][d]; one 16-lane group per (s, h) row of D <= 128.
template <int R>
struct BwdHelperPtrs {
    const __nv_bfloat16 *o[R], *dout[R];
    float *delta[R];
    const float *acc[R];
    __nv_bfloat16 *dq[R];
};

// (one launch for every rank: blockIdx.y = rank)
template <int R>
__global__ void __launch_bounds__(256) bwd_delta_kernel(const __grid_constant__ BwdHelperPtrs<R> hp, int Bl, int S, int H,
                                                        int D) {
    const __nv_bfloat16 *__restrict__ o = hp.o[blockIdx.y];
    const __nv_bfloat16 *__restrict__ dout = hp.dout[blockIdx.y];
    float *__restrict__ delta = hp.delta[blockIdx.y];
    constexpr int lanes = 16;                           // threads per row (16 bytes each; D / 8 of them have data)
    const long long rows = (long long)Bl * S * H;
    const long long gid = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    const long long rowi = gid / lanes;
    const int part = (int)(gid % lanes);
    float acc = 0.f;
    if (rowi < rows && part * 8 < D) {
        const uint4 a = *reinterpret_cast<const uint4 *>(o + rowi * D + part * 8);
        const uint4 b = *reinterpret_cast<const uint4 *>(dout + rowi * D + part * 8);
        const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc += __uint_as_float(av[i] << 16) * __uint_as_float(bv[i] << 16);
            acc += __uint_as_float(av[i] & 0xffff0000u) * __uint_as_float(bv[i] & 0xffff0000u);
        }
    }
    for (int off = lanes / 2; off > 0; off >>= 1) acc += __shfl_down_sync(0xffffffffu, acc, off, lanes);
    if (rowi < rows && part == 0) {
        const long long h = rowi % H, s = (rowi / H) % S, bl = rowi / ((long long)H * S);
        delta[(bl * H + h) * S + s] = acc;
    }
}

// bf16(dQ accumulator), 8 elements per thread.
template <int R>
__global__ void __launch_bounds__(256) bwd_dq_convert_kernel(const __grid_constant__ BwdHelperPtrs<R> hp, long long n8) {
    const float *__restrict__ acc = hp.acc[blockIdx.y];
    __nv_bfloat16 *__restrict__ out = hp.dq[blockIdx.y];
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= n8) return;
    const float4 a = reinterpret_cast<const float4 *>(acc)[2 * i], b = reinterpret_cast<const float4 *>(acc)[2 * i + 1];
    uint4 o;
    o.x = pack_bf16x2(a.x, a.y); o.y = pack_bf16x2(a.z, a.w);
    o.z = pack_bf16x2(b.x, b.y); o.w = pack_bf16x2(b.z, b.w);
    reinterpret_cast<uint4 *>(out)[i] = o;
}

size_t bwd_acc_bytes(const basp_plan *p) { return (size_t)p->Bl * p->S * p->Hq_l * p->D * sizeof(float); }
size_t bwd_delta_bytes(const basp_plan *p) { return (((size_t)p->Bl * p->Hq_l * p->S * sizeof(float)) + 255) & ~(size_t)255; }

}  // namespace
