// Forward with capped scores, a bias by distance, or both (attn_masked_fwd.cu has the mathematics and the parameters).  Shaping the scores in
// front of the exponentials left the SM waiting in the plain kernel's form, two softmax warpgroups with 128 columns of a row a thread: two
// warps a scheduler do not hide the latencies, and a loop over 128 columns does not fit the instruction cache beside the other
// warps' code.  Here four warpgroups have 64 columns of a row each, and rescale and store as many columns of O themselves.
//
//   kForm 0  a cap up to 55.  A capped score is bounded, so the exponentials of a row are taken against a constant (0, or the bias of
//            its nearest key): no running maximum, nothing to rescale, the halves of a row are independent.
//   kForm 1  no cap: the running reference of the plain kernel.  The halves of a row tell each other their maximum at every step,
//            through shared memory.  The maximum is taken over raw scores and a bound on the bias of the half, which is at most 63
//            |slope| above what any of its keys has: a reference that is up to 2^96 too large leaves the exponentials ordinary
//            numbers (24 bits above 2^-126).  Steeper slopes, and a diagonal tile with visible keys behind the row, are shaped in place.
//   kForm 2  a wider cap: 2^(cap log2(e)) leaves too little of fp32's range to do without a maximum; always shaped in place.
//
//   warps  0-15  softmax of query tile warp / 8, columns 64 (warp / 4 % 2) .. + 63 of its rows, and the epilogue of as many columns of O
//   warp  16     TMA producer, 17 and 18 MMA issuers (S = Q K^T, O += P V), as in the plain kernel
// TMEM: S | P_0 P_1 | O_0 | O_1 as there.  Registers: 104 a thread for the softmax, 56 for the rest, of the 96 that all are launched with.
// 16K causal tokens, 32/8 heads of 128 (plain scores 1.55-1.7 ms): cap 50 2.05-2.1 ms, a bias 2.3-2.5, both 2.3, a cap that most tiles reach 3.3; with two
// warpgroups cap 50 2.49 ms (then with a polynomial of four terms; four warpgroups 1.97).
#pragma once

constexpr int kSfThreads = 640;
constexpr int kSfProducer = 16, kSfIssueS = 17, kSfIssueO = 18;

struct SfShared {
    uint64_t q_full, q_empty;
    uint64_t kv_full[kMfStages], kv_empty[kMfStages];
    uint64_t s_free, pv_done[2];
    uint64_t s_full[2], p_full[2], o_final[2], o_free[2], l_full[2], m_full[2];
    float l[2][2][2][kTile];         // [item parity][tile][half][row]
    float m[2][2][2][kTile];         // [step parity][tile][half][row]: maxima of the halves
    uint32_t tmem_base;
    int abort_flag;
};

#define SF_WAIT(bar, parity, role, detail)                                     \
    do {                                                                        \
        if (!mbar_wait((bar), (parity), &sh.abort_flag, (role) >= 30 && (role) < 40 ? kMfSleepNs : 0)) { \
            sh.abort_flag = 1;                                                  \
            report(p.status, 7, (role), (detail));                              \
            goto sf_done;                                                       \
        }                                                                       \
    } while (0)

template <int D, int R, int kForm, bool kBias>
__global__ void __launch_bounds__(kSfThreads, 1) attn_shaped_fwd_kernel(const __grid_constant__ MaskedFwdParams<R> p) {
    constexpr int kSlabs = D / 64, kHalf = kTile / 2;
    constexpr int kTileBytes = kTile * D * 2;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sQ = smem;                                // 2 tiles
    uint8_t *sKV = smem + 2 * kTileBytes;              // kMfStages tiles
    __shared__ SfShared sh;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

    if (tid == 0) {
        mbar_init(&sh.q_full, 1);
        mbar_init(&sh.q_empty, 1);
        for (int i = 0; i < kMfStages; ++i) { mbar_init(&sh.kv_full[i], 1); mbar_init(&sh.kv_empty[i], 1); }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&sh.s_full[t], 1);
            mbar_init(&sh.p_full[t], 8);
            mbar_init(&sh.o_final[t], 1);
            mbar_init(&sh.o_free[t], 8);
            mbar_init(&sh.l_full[t], 8);
            mbar_init(&sh.m_full[t], 8);
            mbar_init(&sh.pv_done[t], 1);
        }
        mbar_init(&sh.s_free, 8);
        sh.abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == kSfProducer) { tmem_alloc(&sh.tmem_base, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    wait_previous_kernel();        // (nothing of another kernel's was touched up to here)
    allow_next_kernel();

    if (warp < 16) {
        // =============================================================== softmax of half a row of query tile t
        reg_inc<104>();
        const int t = warp >> 3, half = (warp >> 2) & 1;
        const int row = tid & 127;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t S_a = tmem + kHalf * half + lane_addr;
        const uint32_t P_t = tmem + 128 + 64 * t + 32 * half + lane_addr;
        uint32_t it_cnt = 0, ep_cnt = 0;
        MfItem item;
        for (int round = 0; mf_get_item(p, round, item); ++round) {
            const int qt = 2 * item.block + t, begin = t ? item.t[1].begin : item.t[0].begin, end = t ? item.t[1].end : item.t[0].end;
            const int full = t ? item.t[1].full : item.t[0].full, full_end = t ? item.t[1].full_end : item.t[0].full_end;
            if (qt >= p.n_tiles) continue;
            const int s_pos = qt * kTile + row;
            const bool in_seq = s_pos < p.S;
            __nv_bfloat16 *dst = p.o[item.r] + (((size_t)item.bl * p.S + s_pos) * p.Hq_l + item.h) * p.Dg;
            if (begin >= end) {                                  // no row of the tile sees a key
                if (half == 0 && in_seq) {
                    if (p.has_lse) p.lse[item.r][((size_t)item.bl * p.Hq_l + item.h) * p.S + s_pos] = -INFINITY;
                    for (int c = 0; c < p.Dg; c += 8) *reinterpret_cast<uint4 *>(dst + c) = make_uint4(0, 0, 0, 0);
                }
                continue;
            }
            // keys [lo, hi) of this thread's row
            int lo = 0, hi = 0;
            if (p.score.range) {
                const int2 range = ld_written(p.score.range + ((size_t)item.seq * p.n_tiles + qt) * kTile + row);
                lo = range.x;
                hi = range.y;
            } else if (in_seq) {
                hi = p.causal ? s_pos + 1 : p.S;
            }
            [[maybe_unused]] const float slope = kBias ? ld_written(p.score.slopes + (item.r % p.K) * p.Hq_l + item.h) * 1.4426950408889634f : 0.f;
            [[maybe_unused]] const bool steep = kForm == 2 || fabsf(slope) * (float)(kHalf - 1) > 96.f;
            float ref = kForm == 0 ? 0.f : -INFINITY;
            if constexpr (kForm == 0 && kBias) {
                // |z| is at most the cap (80 in log2 units for this form) against the bias of the row's nearest key (of its furthest, for
                // a negative slope): the largest exponential of the row is an ordinary number, and no other overflows
                const int dist = slope >= 0.f ? max(max(lo - s_pos, s_pos - hi + 1), 0) : max(s_pos - lo, hi - 1 - s_pos);
                if (hi > lo) ref = -slope * (float)dist;
            }
            float l_run = 0.f;
            for (int j = begin; j < end; ++j, ++it_cnt) {
                SF_WAIT(&sh.s_full[t], it_cnt & 1, 10 + t, j);
                tc_fence_after();
                uint32_t s[kHalf];
                tmem_ld_x32(S_a + 0, *reinterpret_cast<uint32_t(*)[32]>(&s[0]));
                tmem_ld_x32(S_a + 32, *reinterpret_cast<uint32_t(*)[32]>(&s[32]));
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.s_free);       // the scores are in registers: the other tile's Q.K^T may overwrite S
                const int key0 = j * kTile + kHalf * half;
                const bool edge = j < full || j >= full_end;
                // bias of key i: sl i + base, on either side of the row; in the diagonal tile keys behind the row (`fold`) have the other sign
                [[maybe_unused]] float sl = 0.f, base = 0.f;
                [[maybe_unused]] bool fold = false;
                if constexpr (kBias) {
                    sl = j <= qt ? slope : -slope;
                    base = -sl * (float)(s_pos - key0);
                    fold = j == qt && __any_sync(0xffffffffu, min(hi - j * kTile, kTile) - 1 > row);
                }
                [[maybe_unused]] bool far = false;           // kForm 0: some score is not small against the cap
                if constexpr (kForm == 0) {
                    float top[2] = {0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < kHalf; i += 4)
#pragma unroll
                        for (int k = 0; k < 2; ++k) top[k] = max3_abs(top[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
                    const float largest = fmaxf(top[0], top[1]);
                    far = fold || __any_sync(0xffffffffu, largest > p.score.near_limit);
                    // -infinity stands for a hidden key from here on: a product beyond fp32 is the cap's lower end instead
                    if (__builtin_expect(far && __any_sync(0xffffffffu, largest == INFINITY), 0)) {
#pragma unroll
                        for (int i = 0; i < kHalf; ++i)
                            if (s[i] == 0xff800000u) s[i] = 0xff7fffffu;
                    }
                }
                [[maybe_unused]] const bool placed = kForm != 0 && (steep || fold);
                if constexpr (kForm != 0)
                    if (__builtin_expect(placed, kForm == 2)) shape_scores<kForm == 2, kBias>(s, p.score, p.scale_log2, slope, s_pos - key0);
                if (__builtin_expect(edge, 0)) {              // keys outside of [lo, hi) are hidden
                    const int first = lo - key0, past = hi - key0;
                    if (__any_sync(0xffffffffu, first > 0)) {
#pragma unroll
                        for (int i = 0; i < kHalf; ++i)
                            if (i < first) s[i] = 0xff800000u;   // -inf
                    }
                    if (__any_sync(0xffffffffu, past < kHalf)) {
#pragma unroll
                        for (int i = 0; i < kHalf; ++i)
                            if (i >= past) s[i] = 0xff800000u;
                    }
                }
                [[maybe_unused]] float alpha = 1.f;
                if constexpr (kForm != 0) {
                    float top[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) top[k] = max3(__uint_as_float(s[k]), __uint_as_float(s[4 + k]), __uint_as_float(s[8 + k]));
#pragma unroll
                    for (int i = 12; i + 7 < kHalf; i += 8)
#pragma unroll
                        for (int k = 0; k < 4; ++k) top[k] = max3(top[k], __uint_as_float(s[i + k]), __uint_as_float(s[i + 4 + k]));
#pragma unroll
                    for (int k = 0; k < 4; ++k) top[k] = fmaxf(top[k], __uint_as_float(s[60 + k]));
                    float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                    if (!placed && mx != -INFINITY) {
                        mx *= p.scale_log2;
                        if constexpr (kBias) mx += fmaxf(base, fmaf(sl, (float)(kHalf - 1), base));
                    }
                    sh.m[it_cnt & 1][t][half][row] = mx;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.m_full[t]);
                    SF_WAIT(&sh.m_full[t], it_cnt & 1, 12 + t, j);
                    mx = fmaxf(mx, sh.m[it_cnt & 1][t][half ^ 1][row]);
                    if (mx > ref + kMfRescale) { alpha = exp2_approx(ref - mx); ref = mx; }
                    l_run *= alpha;
                }
                const float sub = ref == -INFINITY ? 0.f : ref;        // no key yet: every exponential is exp2(-inf) = 0
                uint64_t sum2[2] = {0ull, 0ull};
                // kKind: 0 capped by the polynomial, 1 by the formula that holds everywhere (and -inf where it stands), 2 raw, 3 in log2 units already
                auto exp_row = [&](auto kind_tag, auto edge_tag) {
                    constexpr int kKind = decltype(kind_tag)::value;
                    constexpr bool kRamp = kBias && kKind != 3;
                    [[maybe_unused]] constexpr bool kEdge = decltype(edge_tag)::value;
                    [[maybe_unused]] const uint64_t minus2 = both(-sub), scale2 = both(p.scale_log2);
                    [[maybe_unused]] uint64_t ramp[2], block = 0;         // the bias of pair i as ramp + block: no constants in the code
                    if constexpr (kRamp) {
                        ramp[0] = pack_f2(0.f, sl);
                        ramp[1] = pack_f2(2.f * sl, 3.f * sl);
                    }
                    [[maybe_unused]] const float most = p.score.near_limit * p.score.near_limit;
#pragma unroll
                    for (int i = 0; i < kHalf; i += 2) {
                        const uint64_t s2 = pack_f2(__uint_as_float(s[i]), __uint_as_float(s[i + 1]));
                        [[maybe_unused]] uint64_t off = minus2;
                        if constexpr (kRamp) {
                            if (i % 4 == 0) block = both(fmaf(sl, (float)i, base - sub));
                            off = add2(ramp[(i >> 1) & 1], block);
                        }
                        uint64_t x2;
                        if constexpr (kKind == 0) {
                            uint64_t y = mul2(s2, s2);
                            if constexpr (kEdge) {                          // -inf: a finite positive q, and -inf again times it
                                float y0, y1;
                                unpack_f2(y, y0, y1);
                                y = pack_f2(fminf(y0, most), fminf(y1, most));
                            }
                            x2 = kBias ? fma2(s2, cap_near_q(y, p.score), off) : mul2(s2, cap_near_q(y, p.score));
                        } else if constexpr (kKind == 1) {
                            // c - 2 c / (exp(2x) + 1); the bound keeps exp(2x) finite
                            float w0, w1;
                            unpack_f2(mul2(s2, both(p.score.cap_in * 2.8853900817779268f)), w0, w1);
                            unpack_f2(add2(pack_f2(exp2_approx(w0 > 64.f ? 64.f : w0), exp2_approx(w1 > 64.f ? 64.f : w1)), both(1.f)), w0, w1);
                            x2 = fma2(pack_f2(rcp_approx(w0), rcp_approx(w1)), both(-2.f * p.score.cap_out), both(p.score.cap_out));
                            if constexpr (kBias) x2 = add2(x2, off);
                            float x0, x1;
                            unpack_f2(x2, x0, x1);
                            x2 = pack_f2(s[i] == 0xff800000u ? -INFINITY : x0, s[i + 1] == 0xff800000u ? -INFINITY : x1);
                        } else if constexpr (kKind == 2) {
                            x2 = fma2(s2, scale2, off);
                        } else {
                            x2 = add2(s2, off);
                        }
                        float x0, x1;
                        unpack_f2(x2, x0, x1);
                        if constexpr (kBias && kKind == 1) {
                            if (fold) {          // -slope |i - at| in the place of slope (i - at)
                                const float at = (float)(s_pos - key0);
                                x0 = fmaf(-2.f * slope, fmaxf((float)i - at, 0.f), x0);
                                x1 = fmaf(-2.f * slope, fmaxf((float)(i + 1) - at, 0.f), x1);
                            }
                        }
                        const float e0 = exp2_approx(x0), e1 = exp2_approx(x1);
                        sum2[(i >> 1) & 1] = add2(sum2[(i >> 1) & 1], pack_f2(e0, e1));
                        s[i >> 1] = pack_bf16x2(e0, e1);
                    }
                };
                if constexpr (kForm == 0) {
                    if (__builtin_expect(far, 0)) exp_row(std::integral_constant<int, 1>{}, std::true_type{});
                    else if (__builtin_expect(edge, 0)) exp_row(std::integral_constant<int, 0>{}, std::true_type{});
                    else exp_row(std::integral_constant<int, 0>{}, std::false_type{});
                } else if constexpr (kForm == 1) {
                    if (__builtin_expect(placed, 0)) exp_row(std::integral_constant<int, 3>{}, std::false_type{});
                    else exp_row(std::integral_constant<int, 2>{}, std::false_type{});
                } else {
                    exp_row(std::integral_constant<int, 3>{}, std::false_type{});
                }
                float ra, rb;
                unpack_f2(add2(sum2[0], sum2[1]), ra, rb);
                l_run += ra + rb;
                // the previous P_t V has read P_t before this step's replaces it
                if (it_cnt > 0) { SF_WAIT(&sh.pv_done[t], (it_cnt - 1) & 1, 14 + t, j); tc_fence_after(); }
                if constexpr (kForm != 0) {
                    // rare after a row's first tiles: this half's columns of O against the new reference
                    if (j > begin && !__all_sync(0xffffffffu, alpha == 1.f)) {
                        const uint32_t O_t = tmem + 256 + 128 * t + (D / 2) * half + lane_addr;
#pragma unroll 1
                        for (int c = 0; c < D / 2; c += 16) {
                            uint32_t rr[16];
                            tmem_ld_x16(O_t + c, rr);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) rr[i] = __float_as_uint(__uint_as_float(rr[i]) * alpha);
                            tmem_st_x16(O_t + c, rr);
                        }
                    }
                }
                tmem_st_x32(P_t, *reinterpret_cast<const uint32_t(*)[32]>(&s[0]));
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_full[t]);
            }
            // ---- the row's sum, LSE, and this half's columns of O
            sh.l[ep_cnt & 1][t][half][row] = l_run;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.l_full[t]);
            SF_WAIT(&sh.l_full[t], ep_cnt & 1, 16 + t, 0);
            const float l = sh.l[ep_cnt & 1][t][0][row] + sh.l[ep_cnt & 1][t][1][row];
            const float inv_l = l == 0.f ? 0.f : 1.f / (hi - lo == 1 ? round_bf16(l) : l);  // no key: P was zero throughout; one key: as there
            if (half == 0 && p.has_lse && in_seq)
                p.lse[item.r][((size_t)item.bl * p.Hq_l + item.h) * p.S + s_pos] = l == 0.f ? -INFINITY : ref * 0.6931471805599453f + logf(l);
            SF_WAIT(&sh.o_final[t], ep_cnt & 1, 18 + t, 0);
            ++ep_cnt;
            tc_fence_after();
            const uint32_t O_t = tmem + 256 + 128 * t + lane_addr;
#pragma unroll 1
            for (int c = half * (D / 2); c < (half + 1) * (D / 2) && c < p.Dg; c += 32) {
                uint32_t rr[32];
                tmem_ld_x32(O_t + c, rr);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    uint4 o4;
                    o4.x = pack_bf16x2(__uint_as_float(rr[i + 0]) * inv_l, __uint_as_float(rr[i + 1]) * inv_l);
                    o4.y = pack_bf16x2(__uint_as_float(rr[i + 2]) * inv_l, __uint_as_float(rr[i + 3]) * inv_l);
                    o4.z = pack_bf16x2(__uint_as_float(rr[i + 4]) * inv_l, __uint_as_float(rr[i + 5]) * inv_l);
                    o4.w = pack_bf16x2(__uint_as_float(rr[i + 6]) * inv_l, __uint_as_float(rr[i + 7]) * inv_l);
                    if (in_seq && c + i < p.Dg) *reinterpret_cast<uint4 *>(dst + c + i) = o4;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.o_free[t]);
        }
    } else {
        reg_dec<56>();
        if (warp == kSfProducer) {
            // =========================================================== TMA producer (lane 0 issues)
            uint32_t kv_it = 0, item_n = 0;
            MfItem item;
            for (int round = 0; mf_get_item(p, round, item); ++round) {
                if (item.j0 >= item.j1) continue;
                SF_WAIT(&sh.q_empty, (item_n & 1) ^ 1, 30, round);
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
                        SF_WAIT(&sh.kv_empty[slot], ph ^ 1, 31, j);
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
        } else if (warp == kSfIssueS) {
            // =========================================================== S = Q_t K_j^T (lane 0 issues)
            const uint32_t idesc_qk = make_idesc_bf16(kTile, kTile, false, false);
            uint32_t item_n = 0, qk_cnt = 0, kv_base = 0;     // K_j of the item at ring index kv_base + 2 (j - j0)
            MfItem item;
            const uint64_t desc_k = make_smem_desc_sw128(0, 16, 1024);        // K-major operands (Q, K)
            const uint32_t q_addr16 = smem_u32(sQ) >> 4, kv_addr16 = smem_u32(sKV) >> 4;
            for (int round = 0; mf_get_item(p, round, item); ++round) {
                if (item.j0 >= item.j1) continue;
                SF_WAIT(&sh.q_full, item_n & 1, 40, round);
                ++item_n;
                for (int j = item.j0; j < item.j1; ++j) {
                    const uint32_t idx = kv_base + 2 * (j - item.j0), slot = idx % kMfStages;
                    SF_WAIT(&sh.kv_full[slot], (idx / kMfStages) & 1, 41, j);
                    tc_fence_after();
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (j < item.t[t].begin || j >= item.t[t].end) continue;
                        // score tile number q may only follow the hand-over of q - 1 to its softmax warps
                        if (qk_cnt > 0) { SF_WAIT(&sh.s_free, (qk_cnt - 1) & 1, 48, j); tc_fence_after(); }
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
        } else if (warp == kSfIssueO) {
            // =========================================================== O_t += P_t V_j (lane 0 issues)
            const uint32_t idesc_pv = make_idesc_bf16(kTile, D, false, true);
            uint32_t it_cnt[2] = {0, 0}, ep_cnt[2] = {0, 0}, kv_base = 0;     // V_j at ring index kv_base + 2 (j - j0) + 1
            MfItem item;
            const uint64_t desc_v = make_smem_desc_sw128(0, 16384, 1024);     // MN-major operand (V)
            const uint32_t kv_addr16 = smem_u32(sKV) >> 4;
            for (int round = 0; mf_get_item(p, round, item); ++round) {
                if (item.j0 >= item.j1) continue;
                for (int j = item.j0; j < item.j1; ++j) {
                    const uint32_t idx = kv_base + 2 * (j - item.j0) + 1, slot = idx % kMfStages;
                    SF_WAIT(&sh.kv_full[slot], (idx / kMfStages) & 1, 42, j);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (j < item.t[t].begin || j >= item.t[t].end) continue;
                        if (j == item.t[t].begin) SF_WAIT(&sh.o_free[t], (ep_cnt[t] & 1) ^ 1, 43 + t, round);
                        SF_WAIT(&sh.p_full[t], it_cnt[t] & 1, 45 + t, j);
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

sf_done:
    tc_fence_before();
    __syncthreads();
    if (sh.abort_flag) {
        // let copies that are still in flight land before the shared memory is given back
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) { }
        __syncthreads();
    }
    if (warp == kSfProducer) tmem_dealloc(tmem, 512);
}

#undef SF_WAIT
