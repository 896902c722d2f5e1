// The activations that a layer's backward pass needs (Q, K, V and O, sequence-sharded), kept in 8 bits between the passes.
//
//   one head vector x[D]:  top = max |x_i|,  scale = top / 127,  code_i = round_half_even(x_i (127 / top))
//   brought back as        x'_i = bf16(code_i scale):  off by at most scale / 2 and the rounding to bf16
//
// A vector with an infinity or a NaN gets the scale NaN (all of it comes back as NaN: the failure stays visible); one whose
// top is below 2^-100 is stored as zeros (127 / top would leave the range of fp32).
// A rank's checkpoint is one buffer: the codes of Q, K, V, O, each in the order of its shard [Bl][T][H][D], then their scales
// (fp32 [Bl][T][H] each, every section at a multiple of 16 bytes).
//
// Both kernels are HBM-bound: packing reads 2 bytes and writes 1 per element, the way back (which is also the exchange from
// sequence- to head-sharded that the backward pass needs anyway) reads 1 and writes 2.  The unit of a thread is 16 elements:
// 32 bytes of bf16, 16 bytes of codes.
#include <cuda_bf16.h>

#include <utility>

#include "common.cuh"
#include "spans.h"

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                    // units in flight per thread
constexpr int kTensors = 4;                   // Q, K, V, O

struct Words8 { uint32_t w[8]; };             // 16 bf16

// kWide: one 256-bit access (the buffers lie on multiples of 32 bytes), else two of 128 bits.
template <bool kWide>
__device__ __forceinline__ Words8 load_unit(const char *p) {
    Words8 v;
    if constexpr (kWide) {
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]),
                       "=r"(v.w[7]) : "l"(p));
    } else {
        const uint4 a = __ldg((const uint4 *)p), b = __ldg((const uint4 *)p + 1);
        v.w[0] = a.x; v.w[1] = a.y; v.w[2] = a.z; v.w[3] = a.w; v.w[4] = b.x; v.w[5] = b.y; v.w[6] = b.z; v.w[7] = b.w;
    }
    return v;
}
template <bool kWide>
__device__ __forceinline__ void store_unit(char *p, const Words8 &v) {
    if constexpr (kWide) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     :: "l"(p), "r"(v.w[0]), "r"(v.w[1]), "r"(v.w[2]), "r"(v.w[3]), "r"(v.w[4]), "r"(v.w[5]), "r"(v.w[6]),
                        "r"(v.w[7]) : "memory");
    } else {
        ((uint4 *)p)[0] = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
        ((uint4 *)p)[1] = make_uint4(v.w[4], v.w[5], v.w[6], v.w[7]);
    }
}

struct CkptTensor {
    uint64_t codes[2], scales[2];             // byte offsets in a rank's checkpoint; [1] where the rank is a group's last
    uint32_t heads;
    uint32_t row_u, run_u;                    // units per token row, and per run of one head-side rank
    uint32_t rep;                             // head-side ranks that receive each run
    uint32_t chunk_begin, chunks_per_shard;
    FastDiv div_row, div_run;
};

// R: room for ranks (8 or BASP_MAX_RANKS; a launch takes longer the larger its parameters)
template <int R>
struct CkptParams {
    char *ckpt[R];
    const char *wide[kTensors][R];            // bf16 shards: sequence side (pack), head side (way back)
    CkptTensor t[kTensors];
    uint32_t K, T, T_last, S, Bl, D, vec_u;       // vec_u: units per head vector = D / 16
    FastDiv div_T, div_T_last, div_vec;
};

struct Where {
    int tensor;
    uint32_t rank, chunk, local;
    bool last;
};
template <int R>
__device__ __forceinline__ Where where(const CkptParams<R> &p) {
    Where w;
    uint32_t c = blockIdx.x;
    w.tensor = 0;
    while (w.tensor + 1 < kTensors && c >= p.t[w.tensor + 1].chunk_begin) ++w.tensor;
    const CkptTensor &t = p.t[w.tensor];
    c -= t.chunk_begin;
    w.rank = c / t.chunks_per_shard;
    w.chunk = c - w.rank * t.chunks_per_shard;
    w.local = w.rank % p.K;
    w.last = w.local == p.K - 1;
    return w;
}

// The largest of the N lanes that hold a vector, in all of them; `lane`: this one's place among them.
template <int N>
__device__ __forceinline__ uint32_t group_max(uint32_t v, int lane) {
    if constexpr ((N & (N - 1)) == 0) {
#pragma unroll
        for (int o = N / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
        return v;
    } else {
#pragma unroll
        for (int o = N > 4 ? 4 : 2; o > 0; o >>= 1) {
            const uint32_t far = __shfl_down_sync(0xffffffffu, v, o);
            if (lane + o < N) v = max(v, far);
        }
        return __shfl_sync(0xffffffffu, v, (threadIdx.x & 31) - lane);
    }
}

// N = D / 16 lanes hold a head vector, 16 elements each; a warp holds 32 / N vectors.
template <int N, bool kWide, int R>
__global__ void __launch_bounds__(kThreads) ckpt_pack_kernel(const __grid_constant__ CkptParams<R> p) {
    constexpr uint32_t kPerWarp = 32 / N, kGroups = kThreads / 32 * kPerWarp;
    const Where at = where(p);
    const CkptTensor &t = p.t[at.tensor];
    const uint32_t warp_lane = threadIdx.x & 31, vec = warp_lane / N, lane = warp_lane - vec * N, group = threadIdx.x / 32 * kPerWarp + vec;
    const bool mine = vec < kPerWarp;
    const uint32_t vectors = p.Bl * (at.last ? p.T_last : p.T) * t.heads;
    const uint32_t v0 = at.chunk * kGroups * kUnroll + group;
    const char *src = p.wide[at.tensor][at.rank];
    char *codes = p.ckpt[at.rank] + t.codes[at.last];
    float *scales = reinterpret_cast<float *>(p.ckpt[at.rank] + t.scales[at.last]);
    Words8 x[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const uint32_t v = v0 + i * kGroups;
        if (v < vectors && mine) x[i] = load_unit<kWide>(src + ((uint64_t)v * N + lane) * 32);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i].w[e] = 0;
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const uint32_t v = v0 + i * kGroups;
        // the magnitudes' bit patterns order like the magnitudes, infinities and NaN above all numbers
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = __vmaxu2(top, x[i].w[e] & 0x7fff7fffu);
        top = max(top & 0xffffu, top >> 16);
        top = group_max<N>(top, (int)lane);
        const float amax = __uint_as_float(top << 16);
        const bool zero = amax < 7.888609052210118e-31f;             // 2^-100
        const float inv = zero ? 0.f : __fdiv_rn(127.f, amax);
        const float scale = top >= 0x7f80u ? __uint_as_float(0x7fc00000u) : (zero ? 0.f : __fdiv_rn(amax, 127.f));
        uint32_t out[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            // adding 1.5 * 2^23 leaves the nearest whole number (ties to even) in the low bits, in two's complement
            uint32_t b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = x[i].w[2 * q + e / 2];
                const float f = __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
                b[e] = __float_as_uint(__fadd_rn(__fmul_rn(f, inv), 12582912.f));
            }
            out[q] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        }
        if (v < vectors && mine) {
            *reinterpret_cast<uint4 *>(codes + ((uint64_t)v * N + lane) * 16) = make_uint4(out[0], out[1], out[2], out[3]);
            if (lane == 0) scales[v] = scale;
        }
    }
}

// The way back: walk the codes in memory order, write every run of a token's heads to the rank that owns them.
template <bool kWide, int R>
__global__ void __launch_bounds__(kThreads) ckpt_to_heads_kernel(const __grid_constant__ CkptParams<R> p) {
    const Where at = where(p);
    const CkptTensor &t = p.t[at.tensor];
    const uint32_t Tr = at.last ? p.T_last : p.T;
    const FastDiv div_Tr = at.last ? p.div_T_last : p.div_T;
    const uint32_t units = p.Bl * Tr * t.row_u;
    const uint32_t u0 = at.chunk * (kThreads * kUnroll) + threadIdx.x;
    const uint32_t first = at.rank - at.local;                       // of the rank's group
    const char *codes = p.ckpt[at.rank] + t.codes[at.last];
    const float *scales = reinterpret_cast<const float *>(p.ckpt[at.rank] + t.scales[at.last]);
    uint4 code[kUnroll];
    float scale[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const uint32_t u = u0 + i * kThreads;
        if (u >= units) continue;
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(code[i].x), "=r"(code[i].y), "=r"(code[i].z), "=r"(code[i].w) : "l"(codes + (uint64_t)u * 16));
        scale[i] = __ldg(scales + fdiv(u, p.div_vec));
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
        const uint32_t u = u0 + i * kThreads;
        if (u >= units) continue;
        const uint32_t tok = fdiv(u, t.div_row), col = u - tok * t.row_u;
        const uint32_t m = fdiv(col, t.div_run), j = col - m * t.run_u;
        const uint32_t bl = fdiv(tok, div_Tr), tt = tok - bl * Tr;
        const uint64_t off = ((uint64_t)(bl * p.S + at.local * p.T + tt) * t.run_u + j) * 32;
        const uint32_t c4[4] = {code[i].x, code[i].y, code[i].z, code[i].w};
        Words8 out;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            // code + 128 as the low byte of 2^23 + code + 128: a byte move and a subtraction, exact
            const uint32_t b = c4[q] ^ 0x80808080u;
            float f[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                f[e] = (__uint_as_float(__byte_perm(b, 0x4b000000u, 0x7440 + e)) - 8388736.f) * scale[i];
            const __nv_bfloat162 lo = __floats2bfloat162_rn(f[0], f[1]), hi = __floats2bfloat162_rn(f[2], f[3]);
            out.w[2 * q] = *reinterpret_cast<const uint32_t *>(&lo);
            out.w[2 * q + 1] = *reinterpret_cast<const uint32_t *>(&hi);
        }
        for (uint32_t c = 0; c < t.rep; ++c)
            store_unit<kWide>(const_cast<char *>(p.wide[at.tensor][first + m * t.rep + c]) + off, out);
    }
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

int heads_of(const basp_plan *p, int tensor) { return tensor == 0 || tensor == 3 ? p->Hq : p->Hkv; }

// Section offsets of a rank with `tokens` tokens per sequence; returns the checkpoint's size.
size_t layout(const basp_plan *p, int tokens, uint64_t (&codes)[kTensors], uint64_t (&scales)[kTensors]) {
    size_t at = 0;
    for (int i = 0; i < kTensors; ++i) {
        codes[i] = at;
        at += up16((size_t)p->Bl * tokens * heads_of(p, i) * p->D);
    }
    for (int i = 0; i < kTensors; ++i) {
        scales[i] = at;
        at += up16((size_t)p->Bl * tokens * heads_of(p, i) * 4);
    }
    return at;
}

// Geometry, chunks and spans of either direction; `units_per_chunk` in head vectors (pack) or units (way back).
template <int R>
int fill(const basp_plan *p, const void *const *ckpt, const void *const *const (&wide)[kTensors], bool pack, CkptParams<R> *prm,
         SpanSet *spans, uint32_t *blocks) {
    if (p->D % 16 != 0 || p->D > 128) return BASP_ERR_UNSUPPORTED;
    if (!ckpt) return BASP_ERR_NULL;
    prm->K = p->K; prm->T = p->T; prm->T_last = p->T_last; prm->S = p->S; prm->Bl = p->Bl; prm->D = p->D;
    prm->vec_u = p->D / 16;
    prm->div_T = make_fastdiv((uint32_t)p->T); prm->div_T_last = make_fastdiv((uint32_t)p->T_last);
    prm->div_vec = make_fastdiv(prm->vec_u);
    uint64_t codes[kTensors], scales[kTensors], codes_last[kTensors], scales_last[kTensors];
    const size_t size = layout(p, p->T, codes, scales), size_last = layout(p, p->T_last, codes_last, scales_last);
    for (int r = 0; r < p->N; ++r) {
        const size_t n = r % p->K == p->K - 1 ? size_last : size;
        BASP_TRY(pack ? spans->add_out(ckpt[r], n) : spans->add_in(ckpt[r], n));
        prm->ckpt[r] = (char *)ckpt[r];
    }
    uint64_t cursor = 0;
    for (int i = 0; i < kTensors; ++i) {
        CkptTensor &t = prm->t[i];
        const int heads = heads_of(p, i);
        t.codes[0] = codes[i]; t.codes[1] = codes_last[i];
        t.scales[0] = scales[i]; t.scales[1] = scales_last[i];
        t.heads = heads;
        t.rep = heads % p->K == 0 ? 1 : p->K / heads;                // a plan has one of the two
        t.run_u = (t.rep > 1 ? 1 : heads / p->K) * prm->vec_u;
        t.row_u = heads * prm->vec_u;
        t.div_row = make_fastdiv(t.row_u); t.div_run = make_fastdiv(t.run_u);
        const uint64_t vectors = (uint64_t)p->Bl * p->T * heads, units = vectors * prm->vec_u;
        const uint64_t head_units = (uint64_t)p->Bl * p->S * t.run_u;
        if (units + kThreads * kUnroll >= (1ull << 31) || head_units >= (1ull << 32)) return BASP_ERR_UNSUPPORTED;
        const uint64_t per_chunk = pack ? (uint64_t)(kThreads / 32 * (32 / prm->vec_u)) * kUnroll : (uint64_t)kThreads * kUnroll;
        const uint64_t chunks = ((pack ? vectors : units) + per_chunk - 1) / per_chunk;
        t.chunk_begin = (uint32_t)cursor;
        t.chunks_per_shard = (uint32_t)chunks;
        cursor += chunks * p->N;
        if (!wide[i]) return BASP_ERR_NULL;
        for (int r = 0; r < p->N; ++r) {
            const size_t bytes = pack ? (size_t)p->Bl * basp_rank_tokens(p, r % p->K) * heads * p->D * 2 : (size_t)head_units * 32;
            BASP_TRY(pack ? spans->add_in(wide[i][r], bytes) : spans->add_out(wide[i][r], bytes));
            prm->wide[i][r] = (const char *)wide[i][r];
        }
    }
    if (cursor >= (1ull << 31)) return BASP_ERR_UNSUPPORTED;
    *blocks = (uint32_t)cursor;
    return spans->overlaps();
}

// 256-bit accesses fault below 32-byte alignment; the interface promises 16.
template <int R>
bool all_on_32(const basp_plan *p, const CkptParams<R> &prm) {
    uintptr_t bits = 0;
    for (int i = 0; i < kTensors; ++i)
        for (int r = 0; r < p->N; ++r) bits |= (uintptr_t)prm.wide[i][r];
    return (bits & 31) == 0;
}

template <int R, int... kN>
void launch_pack(const CkptParams<R> &prm, uint32_t blocks, bool wide, cudaStream_t st, std::integer_sequence<int, kN...>) {
    ((prm.vec_u != kN + 1 ? (void)0
                          : wide ? ckpt_pack_kernel<kN + 1, true, R><<<blocks, kThreads, 0, st>>>(prm)
                                 : ckpt_pack_kernel<kN + 1, false, R><<<blocks, kThreads, 0, st>>>(prm)), ...);
}

template <int R>
int run_pack(const basp_plan *p, const void *const *const (&shards)[kTensors], void *const *ckpt_shards, cudaStream_t st) {
    CkptParams<R> prm;
    SpanSet spans;
    uint32_t blocks = 0;
    BASP_TRY(fill(p, (const void *const *)ckpt_shards, shards, true, &prm, &spans, &blocks));
    const bool wide = all_on_32(p, prm);
    launch_pack(prm, blocks, wide, st, std::make_integer_sequence<int, 8>{});
    BASP_CUDA_TRY(cudaGetLastError());
    basp_count_launch(1);
    return BASP_OK;
}

template <int R>
int run_to_heads(const basp_plan *p, const void *const *ckpt_shards, const void *const *const (&heads)[kTensors], cudaStream_t st) {
    CkptParams<R> prm;
    SpanSet spans;
    uint32_t blocks = 0;
    BASP_TRY(fill(p, ckpt_shards, heads, false, &prm, &spans, &blocks));
    if (all_on_32(p, prm)) ckpt_to_heads_kernel<true, R><<<blocks, kThreads, 0, st>>>(prm);
    else ckpt_to_heads_kernel<false, R><<<blocks, kThreads, 0, st>>>(prm);
    BASP_CUDA_TRY(cudaGetLastError());
    basp_count_launch(1);
    return BASP_OK;
}

}  // namespace

extern "C" size_t basp_ckpt_bytes(const basp_plan *p, int rank) {
    if (!p || rank < 0 || rank >= p->N) return 0;
    uint64_t codes[kTensors], scales[kTensors];
    return layout(p, basp_rank_tokens(p, rank % p->K), codes, scales);
}

extern "C" int basp_ckpt_pack(const basp_plan *p, const void *const *q_seq, const void *const *k_seq, const void *const *v_seq,
                              const void *const *o_seq, void *const *ckpt_shards, void *stream) {
    if (!p) return BASP_ERR_NULL;
    const void *const *const shards[kTensors] = {q_seq, k_seq, v_seq, o_seq};
    return p->N <= 8 ? run_pack<8>(p, shards, ckpt_shards, (cudaStream_t)stream)
                     : run_pack<BASP_MAX_RANKS>(p, shards, ckpt_shards, (cudaStream_t)stream);
}

extern "C" int basp_ckpt_reshard_s2h(const basp_plan *p, const void *const *ckpt_shards, void *const *q_head, void *const *k_head,
                                     void *const *v_head, void *const *o_head, void *stream) {
    if (!p) return BASP_ERR_NULL;
    typedef const void *const *In;
    const In heads[kTensors] = {(In)q_head, (In)k_head, (In)v_head, (In)o_head};
    return p->N <= 8 ? run_to_heads<8>(p, ckpt_shards, heads, (cudaStream_t)stream)
                     : run_to_heads<BASP_MAX_RANKS>(p, ckpt_shards, heads, (cudaStream_t)stream);
}
