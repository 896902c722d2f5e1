// Backward with masked and shaped scores, head dimensions 80 .. 128: the pipeline of attn_bwd_d128.cuh (order of the products, TMEM
// and stages as there; the barriers and the order of issue are written out in both files: a change of one is a change of the other).
// What is different: a key tile's query tiles come from the mask object and may be none; the producer
// stages for every query the window of the tile's keys that it sees, and whether any of it matters; the probabilities carry
// the cap and the bias, and dS the cap's derivative.
#pragma once

template <int R, bool kCap, bool kBias, bool kSmall>
__global__ void __launch_bounds__(kBwdThreads, 1) attn_masked_bwd_d128_kernel(const __grid_constant__ MaskedBwdParams<R> p) {
    constexpr int D = 128;
    // How far the issuing loops are unrolled: the code of all roles together has to stay in the instruction cache (16K causal tokens, 32/8
    // heads of 128, cap 50: 7.0 ms at four, 7.6 in full; without a cap 5.6 in full, 6.1 at four)
    constexpr int kUnroll = kCap ? 4 : 8;
    constexpr int kTileBytes = kT * D * 2;             // 32 KiB: two slabs of [128 rows][64 columns]
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t *sK = smem, *sV = smem + kTileBytes;
    uint8_t *sQ = smem + 2 * kTileBytes;               // 2 stages
    constexpr int kDoStages = 2;
    uint8_t *sdO = smem + 4 * kTileBytes;
    uint8_t *sdS = smem + (4 + kDoStages) * kTileBytes;   // dS^T [key rows][query cols], two 64-column slabs
    float *s_lse = reinterpret_cast<float *>(smem + 7 * kTileBytes);   // [2][128], already times log2(e)
    float *s_delta = s_lse + 2 * kT;                                   // [2][128], already times -scale
    uint16_t *s_win = reinterpret_cast<uint16_t *>(s_delta + 2 * kT);  // [2][128], see stage_stats
    int *s_edge = reinterpret_cast<int *>(s_win + 2 * kT);             // [2]
    BwdBars *bars = reinterpret_cast<BwdBars *>(s_edge + 2);

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

    if (tid == 0) {
        mbar_init(&bars->kv_full, 1); mbar_init(&bars->kv_empty, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars->qdo_full[s], 1);          // Q stage loaded
            mbar_init(&bars->qdo_mma_done[s], 1);      // Q stage free: products (1) and (4) of its step are done
            mbar_init(&bars->stats_full[s], 1);
            mbar_init(&bars->do_full[s], 1);           // dO stage loaded
            mbar_init(&bars->do_free[s], 1);           // dO stage free: products (2) and (3) of its step are done
        }
        mbar_init(&bars->s_full, 1);
        mbar_init(&bars->dp_full, 1);
        mbar_init(&bars->p_ready, kBwdComputeWarps);
        mbar_init(&bars->pds_ready, kBwdComputeWarps);
        mbar_init(&bars->dq_full, 1);
        mbar_init(&bars->dq_read, 4);
        mbar_init(&bars->dkdv_full, 1);
        mbar_init(&bars->dkdv_read, kBwdComputeWarps);
        bars->abort_flag = (smem_u32(smem) & 1023u) ? 1 : 0;
        if (bars->abort_flag) bwd_report(p.status, 4, 0, (int)(smem_u32(smem) & 1023u));
        fence_mbar_init();
    }
    if (warp == kBwdTmaWarp) { tmem_alloc(&bars->tmem_base, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    wait_previous_kernel();        // (nothing of another kernel's was touched up to here)
    allow_next_kernel();
    constexpr uint32_t kColST = 0, kColDP = 128, kColDK = 256, kColDV = 384;
    if (bars->abort_flag) goto bwd_done;

    if (warp < kBwdComputeWarps) {
        // ======================================================================= compute warps
        const int g = warp >> 2;                        // which 32-column quarter of the score tile
        const int row = tid & 127;                      // TMEM lane: key row
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t st_col = tmem + kColST + 32 * g + lane_addr;
        uint32_t it_g = 0, item_n = 0;
        MbItem item;
        for (int round = 0; mb_get_item<kSmall>(p, round, item); ++round) {
            if (item.m0 >= item.n_qt) {                 // no query sees a key of the tile
                store_zeros<kSmall>(p, item, g, row);
                continue;
            }
            for (int hq = 0; hq < mb_heads<kSmall>(p, item); ++hq) {
                const float slope = kBias ? __ldg(p.score.slopes + (item.r % p.K) * p.Hq_l + mb_first_head<kSmall>(p, item) + hq) * 1.4426950408889634f : 0.f;
                for (int m = item.m0; m < item.n_qt; ++m, ++it_g) {
                    const uint32_t stage = it_g & 1, sph = (it_g >> 1) & 1;     // Q stage of the step (row statistics with it)
                    BWD_WAIT(&bars->stats_full[stage], sph, 10, m);             // LSE and Delta of the query tile
                    BWD_WAIT(&bars->s_full, it_g & 1, 11, m);
                    tc_fence_after();
                    uint32_t st[32], dp[32];
                    tmem_ld_x32(st_col, st);
                    tmem_wait_ld();
                    const float *lse_b = s_lse + stage * kT + 32 * g;
                    const float *del_b = s_delta + stage * kT + 32 * g;
                    // P^T = exp2(z^T - LSE), the scores' shape included: needs the scores only.  What stays in st is P^T times the
                    // derivative of the cap
                    {
                        const int dist = (m - item.n) * kT + 32 * g - row;      // position of the first column's query minus the key's
                        const int edge = s_edge[stage];
                        if (edge || (kBias && m == item.n))
                            shaped_probs<kCap, kBias, true>(st, st_col, lse_b, s_win + stage * kT + 32 * g, row, p.score, p.scale_log2, slope, dist, m - item.n);
                        else
                            shaped_probs<kCap, kBias, false>(st, st_col, lse_b, nullptr, row, p.score, p.scale_log2, slope, dist, m - item.n);
                        if (!kBias && __builtin_expect(edge & 2 << g, 0)) drop_singles(st, s_win + stage * kT + 32 * g);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars->p_ready);          // product (3) of this step may start
                    // dS^T = P^T (dP^T scale - Delta scale)
                    BWD_WAIT(&bars->dp_full, it_g & 1, 12, m);
                    tc_fence_after();
                    tmem_ld_x32(tmem + kColDP + 32 * g + lane_addr, dp);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        const float4 d4 = *reinterpret_cast<const float4 *>(del_b + c);
                        const float dl[4] = {d4.x, d4.y, d4.z, d4.w};
                        float dsv[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            dsv[e] = __uint_as_float(st[c + e]) * fmaf(__uint_as_float(dp[c + e]), p.scale, dl[e]);
                        dp[c >> 1] = pack_bf16x2(dsv[0], dsv[1]);
                        dp[(c >> 1) + 1] = pack_bf16x2(dsv[2], dsv[3]);
                    }
                    // dS^T row `row`, query columns 32g..32g+31 = half a 128-byte line of slab g/2 (128-byte swizzle).  The
                    // buffer's last readers, products (5) and (4) of the step before, were complete before dP^T of this
                    // step was (the tensor pipe finishes in issue order).
                    {
                        uint8_t *line = sdS + (g >> 1) * 16384 + row * 128;
#pragma unroll
                        for (int ch = 0; ch < 4; ++ch)
                            *reinterpret_cast<uint4 *>(line + (((4 * (g & 1) + ch) ^ (row & 7)) << 4)) =
                                make_uint4(dp[4 * ch], dp[4 * ch + 1], dp[4 * ch + 2], dp[4 * ch + 3]);
                    }
                    fence_proxy_async_smem();
                    tc_fence_before();                  // the load of dP^T is complete: Y may take dQ
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars->pds_ready);
                }
            }
            // ---- item done: dK_n (quarters 0, 1) / dV_n (quarters 2, 3) to global as bf16, 64 columns per quarter
            BWD_WAIT(&bars->dkdv_full, item_n & 1, 13, item.n);
            tc_fence_after();
            {
                constexpr int kHalf = D / 2;
                const uint32_t col0 = (g < 2 ? kColDK : kColDV) + kHalf * (g & 1);
#pragma unroll
                for (int cc = 0; cc < kHalf / 32; ++cc) {
                    uint32_t rr[32];
                    tmem_ld_x32(tmem + col0 + cc * 32 + lane_addr, rr);
                    tmem_wait_ld();
                    store_kv<kSmall>(p, item, g >= 2, row, kHalf * (g & 1) + cc * 32, rr);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->dkdv_read);
            ++item_n;
        }
    } else if (warp < kBwdTmaWarp) {
        // ======================================================================= dQ drain warps
        // Product (5) leaves dQ_m TRANSPOSED in Y (lane = feature d, column = query row), so a warp's 32 lanes hold 32
        // consecutive features of one query row per register: one red.global.add.f32 per register adds a complete
        // 128-byte line of the fp32 accumulator.  No shared memory, no staging; Y is handed back once its last columns
        // are in registers.
        reg_inc<120>();
        const int wq = warp & 3;
        const uint32_t lane_addr = (uint32_t)(wq * 32) << 16;
        const int d = wq * 32 + lane;                   // this thread's feature
        uint32_t it_g = 0;
        MbItem item;
        for (int round = 0; mb_get_item<kSmall>(p, round, item); ++round) {
            for (int hq = 0; hq < mb_heads<kSmall>(p, item); ++hq) {
                const int h = mb_first_head<kSmall>(p, item) + hq;
                for (int m = item.m0; m < item.n_qt; ++m, ++it_g) {
                    BWD_WAIT(&bars->dq_full, it_g & 1, 14, m);
                    tc_fence_after();
                    if (kSmall && p.direct) {         // the only key tile: dQ as bf16
                        __nv_bfloat16 *to = p.dq[item.r] + (((size_t)item.bl * p.S + (size_t)m * kT) * p.Hq_l + h) * p.Dg + d;
#pragma unroll 1
                        for (int c0 = 0; c0 < kT; c0 += 32) {
                            uint32_t v[32];
                            tmem_ld_x32(tmem + kColDP + c0 + lane_addr, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (d < p.Dg && m * kT + c0 + c < p.S) to[(size_t)(c0 + c) * p.Hq_l * p.Dg] = __float2bfloat16(__uint_as_float(v[c]));
                        }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars->dq_read);
                        continue;
                    }
                    // accumulator element (query row m*128 + c, head h, feature d); a row past the end of the sequence
                    // (ragged last tile) and a feature past the head dimension have none
                    const size_t acc_row = (size_t)p.Hq_l * p.Dg;
                    float *acc = p.dq_accp[item.r] + (((size_t)item.bl * p.S + (size_t)m * kT) * p.Hq_l + h) * p.Dg + d;
                    const int rows_left = d < p.Dg ? p.S - m * kT : 0;          // columns c < rows_left are added
                    auto add_cols = [&](const uint32_t *v, int c0, int n) {
                        if (c0 + n <= rows_left) {
#pragma unroll
                            for (int c = 0; c < n; ++c)
                                asm volatile("red.global.add.f32 [%0], %1;" ::"l"(acc + (size_t)(c0 + c) * acc_row),
                                             "f"(__uint_as_float(v[c])) : "memory");
                        } else {
#pragma unroll
                            for (int c = 0; c < n; ++c)
                                if (c0 + c < rows_left)
                                    asm volatile("red.global.add.f32 [%0], %1;" ::"l"(acc + (size_t)(c0 + c) * acc_row),
                                                 "f"(__uint_as_float(v[c])) : "memory");
                        }
                    };
                    uint32_t v[96], w[32];
                    tmem_ld_x32(tmem + kColDP + lane_addr, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
                    tmem_ld_x32(tmem + kColDP + 32 + lane_addr, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
                    tmem_ld_x32(tmem + kColDP + 64 + lane_addr, *reinterpret_cast<uint32_t(*)[32]>(&v[64]));
                    tmem_wait_ld();
                    add_cols(&v[0], 0, 32);
                    tmem_ld_x32(tmem + kColDP + 96 + lane_addr, w);
                    tmem_wait_ld();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars->dq_read);          // Y is free for the next dP^T
                    add_cols(&v[32], 32, 64);
                    add_cols(w, 96, 32);
                }
            }
        }
    } else {
      reg_dec<40>();       // 16 x 80 (compute) + 4 x 120 (drain) + 4 x 40 = the 24 x 80 registers per lane the CTA was launched with
      if (warp == kBwdTmaWarp) {
        // ======================================================================= TMA producer
        uint32_t it_g = 0, item_n = 0;
        MbItem item;
        for (int round = 0; mb_get_item<kSmall>(p, round, item); ++round) {
            if (item.m0 >= item.n_qt) continue;
            BWD_WAIT(&bars->kv_empty, (item_n & 1) ^ 1, 20, item.n);
            ++item_n;
            if (lane == 0) {
                mbar_arrive_expect_tx(&bars->kv_full, 2 * kTileBytes);
                const int row0 = item.bl * p.S + item.n * kT;
                for (int s = 0; s < 2; ++s) {
                    tma_load_3d(sK + s * 16384, &p.k[item.r], &bars->kv_full, s * 64, item.hkv, row0);
                    tma_load_3d(sV + s * 16384, &p.v[item.r], &bars->kv_full, s * 64, item.hkv, row0);
                }
            }
            for (int hq = 0; hq < mb_heads<kSmall>(p, item); ++hq) {
                const int h = mb_first_head<kSmall>(p, item) + hq;
                for (int m = item.m0; m < item.n_qt; ++m, ++it_g) {
                    const uint32_t stage = it_g & 1, ph = (it_g >> 1) & 1;
                    const int row0 = item.bl * p.S + m * kT;
                    // Q stage (tile and row statistics): free once products (1) and (4) of two steps ago are done, which also
                    // means that the compute warps have finished that step
                    BWD_WAIT(&bars->qdo_mma_done[stage], ph ^ 1, 21, m);
                    if (lane == 0) {
                        mbar_arrive_expect_tx(&bars->qdo_full[stage], kTileBytes);
                        for (int s = 0; s < 2; ++s)
                            tma_load_3d(sQ + stage * kTileBytes + s * 16384, &p.q[item.r], &bars->qdo_full[stage], s * 64, h, row0);
                    }
                    {
                        const MbStats stats = fetch_stats(p, item, h, m, lane);
                        stage_stats(p, item, m, lane, stats, s_lse + stage * kT, s_delta + stage * kT, s_win + stage * kT, s_edge + stage);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars->stats_full[stage]);
                    }
                    // dO stage: free once product (3) of its previous step is done
                    const uint32_t dstage = it_g % kDoStages, dph = (it_g / kDoStages) & 1;
                    BWD_WAIT(&bars->do_free[dstage], dph ^ 1, 22, m);
                    if (lane == 0) {
                        mbar_arrive_expect_tx(&bars->do_full[dstage], kTileBytes);
                        for (int s = 0; s < 2; ++s)
                            tma_load_3d(sdO + dstage * kTileBytes + s * 16384, &p.dout[item.r], &bars->do_full[dstage], s * 64, h, row0);
                    }
                }
            }
        }
      } else if (warp == kBwdMmaWarp) {
        // ======================================================================= MMA issuer
        const uint32_t idesc_kk = make_idesc_bf16(kT, kT, false, false);     // (1) (2): both operands K-major
        const uint32_t idesc_kn = make_idesc_bf16(kT, D, false, true);       // (3) (4): B is MN-major
        const uint32_t idesc_nn = make_idesc_bf16(kT, D, true, true);        // (5): A and B MN-major
        const uint64_t desc_k = make_smem_desc_sw128(0, 16, 1024);
        const uint64_t desc_mn = make_smem_desc_sw128(0, 16384, 1024);
        const uint32_t aK = smem_u32(sK) >> 4, aV = smem_u32(sV) >> 4, aQ = smem_u32(sQ) >> 4,
                       adO = smem_u32(sdO) >> 4, adS = smem_u32(sdS) >> 4;
        uint32_t it_g = 0, item_n = 0;
        MbItem item;
        for (int round = 0; mb_get_item<kSmall>(p, round, item); ++round) {
            if (item.m0 >= item.n_qt) continue;
            const uint32_t steps = (uint32_t)mb_heads<kSmall>(p, item) * (uint32_t)(item.n_qt - item.m0);
            BWD_WAIT(&bars->kv_full, item_n & 1, 30, item.n);
            // (1) S^T = K Q^T of step `it` into X (its last reader, product (3) of step it-1, was issued before)
            auto issue_s = [&](uint32_t it) -> bool {
                const uint32_t stage = it & 1;
                if (!mbar_wait(&bars->qdo_full[stage], (it >> 1) & 1, &bars->abort_flag)) return false;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t q16 = aQ + stage * (kTileBytes >> 4);
#pragma unroll kUnroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t off = ((kk / 4) * 16384 + (kk % 4) * 32) >> 4;
                        mma_ss(tmem + kColST, desc_k | (uint64_t)(aK + off), desc_k | (uint64_t)(q16 + off), idesc_kk, kk > 0);
                    }
                    tc_commit(&bars->s_full);
                }
                return true;
            };
            // (2) dP^T = V dO^T of step `it` into Y, once dQ of step it-1 has left it
            auto issue_dp = [&](uint32_t it) -> bool {
                if (!mbar_wait(&bars->dq_read, (it & 1) ^ 1, &bars->abort_flag)) return false;
                if (!mbar_wait(&bars->do_full[it % kDoStages], (it / kDoStages) & 1, &bars->abort_flag)) return false;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t do16 = adO + (it % kDoStages) * (kTileBytes >> 4);
#pragma unroll kUnroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t off = ((kk / 4) * 16384 + (kk % 4) * 32) >> 4;
                        mma_ss(tmem + kColDP, desc_k | (uint64_t)(aV + off), desc_k | (uint64_t)(do16 + off), idesc_kk, kk > 0);
                    }
                    tc_commit(&bars->dp_full);
                }
                return true;
            };
            // (3) dV += P^T dO of step `it`: A = P^T in X (query index along K: 8 columns per 16 queries, each quarter of
            //     32 queries starts at its own column 32g), B = dO read MN-major.  The first one of an item also waits
            //     until dK / dV of the item before have been stored.  When it is done the dO stage is free.
            auto issue_dv = [&](uint32_t it, bool first) -> bool {
                if (!mbar_wait(&bars->p_ready, it & 1, &bars->abort_flag)) return false;
                if (first && !mbar_wait(&bars->dkdv_read, (item_n & 1) ^ 1, &bars->abort_flag)) return false;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t do16 = adO + (it % kDoStages) * (kTileBytes >> 4);
#pragma unroll kUnroll
                    for (int kk = 0; kk < kT / 16; ++kk)
                        mma_ts(tmem + kColDV, tmem + kColST + (kk / 2) * 32 + (kk % 2) * 8,
                               desc_mn | (uint64_t)(do16 + kk * 128), idesc_kn, kk > 0 ? 1u : (first ? 0u : 1u));
                    tc_commit(&bars->do_free[it % kDoStages]);
                }
                return true;
            };
            bool ok = issue_s(it_g) && issue_dp(it_g);
            if (!ok) { bars->abort_flag = 1; bwd_report(p.status, 3, 31, item.n); goto bwd_done; }
            for (uint32_t j = 0; j < steps; ++j) {
                const uint32_t it = it_g + j, stage = it & 1;
                const uint32_t q16 = aQ + stage * (kTileBytes >> 4);
                ok = issue_dv(it, j == 0);
                if (ok && j + 1 < steps) ok = issue_s(it + 1);
                if (!ok) { bars->abort_flag = 1; bwd_report(p.status, 3, 32, (int)j); goto bwd_done; }
                BWD_WAIT(&bars->pds_ready, it & 1, 33, (int)j);
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t acc0 = j == 0 ? 0u : 1u;
                    // (5) dQ_m^T = K^T dS^T : A = K read MN-major (rows of the result = features), B = the dS^T buffer read
                    //     MN-major (columns = query rows); transposed so that the drain warps add whole lines
#pragma unroll kUnroll
                    for (int kk = 0; kk < kT / 16; ++kk)
                        mma_ss(tmem + kColDP, desc_mn | (uint64_t)(aK + kk * 128), desc_mn | (uint64_t)(adS + kk * 128),
                               idesc_nn, kk > 0);
                    tc_commit(&bars->dq_full);
                    // (4) dK += dS^T Q : A = dS^T from shared memory (K-major: query columns), B = Q MN-major
#pragma unroll kUnroll
                    for (int kk = 0; kk < kT / 16; ++kk) {
                        const uint32_t off = ((kk / 4) * 16384 + (kk % 4) * 32) >> 4;
                        mma_ss(tmem + kColDK, desc_k | (uint64_t)(adS + off), desc_mn | (uint64_t)(q16 + kk * 128),
                               idesc_kn, kk > 0 ? 1u : acc0);
                    }
                    tc_commit(&bars->qdo_mma_done[stage]);        // (1) and (4) of the step are done: its Q stage may be loaded again
                }
                if (j + 1 < steps && !issue_dp(it + 1)) { bars->abort_flag = 1; bwd_report(p.status, 3, 35, (int)j); goto bwd_done; }
            }
            it_g += steps;
            if (lane == 0) {
                tc_commit(&bars->dkdv_full);
                tc_commit(&bars->kv_empty);
            }
            ++item_n;
        }
      }
    }

bwd_done:
    tc_fence_before();
    __syncthreads();
    if (bars->abort_flag) {
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) { }
        __syncthreads();
    }
    if (warp == kBwdTmaWarp) tmem_dealloc(tmem, 512);
}
