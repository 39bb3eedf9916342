// Gated delta rule, reverse scan.  Per chunk, D the adjoint of the state at its END, from the last chunk to the first, dO' = scale dO:
//     beside the chain, one chunk ahead:   X = P^T dO',   Y = (e^G Q)^T dO'   (fp32, through LDS)
//     chain:   dE = X + e^{G_C - G} beta K D,   dV = T^T dE,   D <- e^{G_C} D + Y - K^T (e^G dV)
//     stores of dV and D, one chunk behind
// Two barriers a step: at its start, and when the chain has taken X and Y and the storing waves have taken the step before's D and dV:
// then either side writes the next.
// PRECISE (a call that asks for dS0, which is 32-bit): as in the forward scan; P^T and e^G dO' have remainders as well (dO and Q are exact).
#include "mdn_gdr_ring.h"
#include "mdn_gdr_scan.h"

namespace mdn {

namespace {

// Waves to 16 columns of the chain, as in the forward scan, two for one, backward calls: 68 us for 84 in fp32 (2 x 1 024 tokens, 4 heads, d = 64),
// 919 for 1 223 (8 192 of 16, d = 128), with remainders 49 for 52 (777 tokens, 16 heads, d = 128), 1 369 for 1 455 (32 768).  (Not with 32
// columns, whose LDS is full.)
template <typename T, int NCG, bool PRECISE> constexpr int CW = (sizeof(T) == 4 || PRECISE) && NCG == 1 ? 2 : 1;
// beside the chain, chain, loads, stores
template <typename T, int DK, int NCG, bool PRECISE> constexpr int bwd_waves() {
    return 2 + CW<T, NCG, PRECISE> * NCG + 2 + (gdr_ring<T, DK, NCG>() ? 2 : 0);
}

template <typename T, int DK, int NCG, bool PRECISE>
__global__ __launch_bounds__((bwd_waves<T, DK, NCG, PRECISE>() * 64)) void gdr_scan_bwd_kernel(GdrDims d, GdrScanBwdArgs a, int first) {
    typedef Gd<T> G;
    typedef typename G::Frag Frag;
    typedef Slate<T, DK> SlateS;
    typedef Slate<T, 64> SlateE;
    constexpr int NT = DK / 16, SK = DK / G::KS, S64 = 64 / G::KS, COLS = 16 * NCG, TRI = G::NF * 64 * G::E;
    constexpr int TB = TRI * (int)sizeof(T); // bytes of a triangle
    constexpr bool RING = gdr_ring<T, DK, NCG>(); // otherwise loads between two barriers, not beside the products
    // ring depths: what the chain reads; T^T; what the waves beside it read (there is no room for three of everything); coefficients
    constexpr int D = RING ? kReverseK : 1, DT = RING ? reverse_t(PRECISE) : 1, DQ = RING ? kReverseQ : 1, DC = kReverseCoef;
    constexpr int CWS = CW<T, NCG, PRECISE>, LOADS = 2 + CWS * NCG, STORES = LOADS + 2; // first waves of each kind
    constexpr int SETS = sizeof(T) == 2 ? 2 : 1; // chunks of P^T that a wave beside the chain has asked for
    typedef GLoad<T, DK, true> LoadK;
    typedef GLoad<T, COLS, false> LoadV;
    __shared__ __align__(16) T s_k[D][64 * DK], s_q[DQ][64 * DK], s_do[DQ][64 * COLS], s_t[DT][TRI], s_tl[DT][PRECISE ? TRI : 8];
    __shared__ __align__(16) float s_c[DC][kGdrCoef];
    __shared__ __align__(16) f32x4 s_x[NCG][4][64], s_y[NCG][NT][64];
    __shared__ __align__(16) T s_s[CWS][NCG][SlateS::SIZE], s_sl[NCG][CWS == 2 && PRECISE ? SlateS::SIZE : 8], s_r[NCG * SlateE::SIZE];
    __shared__ __align__(16) Frag s_e[NCG][CWS == 2 ? S64 : 1][64], s_el[NCG][CWS == 2 && PRECISE ? S64 : 1][64]; // dE, from wave to wave
    __shared__ int s_said[NCG][2]; // steps whose half of it is there
    __shared__ __align__(16) int s_touch[2][64];

    const int w = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, kg = lane >> 4;
    int bh, sub;
    xcd_map(first + (int)blockIdx.x, d.dv / COLS, bh, sub);
    if (bh >= d.B * d.H) return;
    const GdrSeq q = gdr_seq(d, bh);
    const int col0 = sub * COLS, N = q.n, last = (q.len - 1) & 63; // last: the last row of the last chunk
    const unsigned rsv = (unsigned)(d.H * d.dv), rsk = (unsigned)(d.Hk * DK);

    // Step n: chunk N - 1 - n on the chain, the one before it (in time) beside it
    auto store = [&](int n, int w2) { // dV, D of step n
        const int r = lane & 15, kg = lane >> 4, m = N - 1 - n;
        const size_t at = (q.v + (size_t)m * 64 * d.H) * d.dv + col0, reach = ((size_t)(n == 0 ? last : 63) * rsv + COLS) * sizeof(T);
        store_tokens<T, NCG, SlateE::LD>(out_rows(static_cast<T *>(a.dv) + at, reach), rsv * (unsigned)sizeof(T), s_r, 32 * w2, 32 * w2, r, kg);
        store_state<T, DK, NCG>(out_rows(static_cast<T *>(a.dstates) + (q.blk + m) * DK * d.dv, (size_t)DK * d.dv * sizeof(T)), s_s[n % CWS], w2, col0, lane);
    };
    // (not with remainders, where the chain is what a step waits for)
    GdrTouch<PRECISE ? 0 : touch_places(2 * DK * (int)sizeof(T) + 2 * TB / 64 + 16, (int)sizeof(T), COLS)> touch;
    auto aim_touch = [&](int w2) {
        touch.aim(sub * 2 + w2, d.dv / COLS * 2, lane);
        const ptrdiff_t row = rsk * sizeof(T), rov = rsv * sizeof(T);
        touch.add(static_cast<const T *>(a.k) + q.k * DK, 64, DK * sizeof(T), row, 64 * row, N, last);
        touch.add(static_cast<const T *>(a.q) + q.k * DK, 64, DK * sizeof(T), row, 64 * row, N, last);
        touch.add(static_cast<const T *>(a.dO) + q.v * d.dv, 64, d.dv * sizeof(T), rov, 64 * rov, N, last);
        auto block = [&](const void *t, int bytes) { touch.add(static_cast<const char *>(t) + q.blk * bytes, 1, bytes, 0, bytes, N, 0); };
        block(a.TT, TB);
        block(a.PT, TB);
        block(a.coef, kGdrCoef * 4);
    };
    if (w >= STORES) {
        const int w2 = w - STORES;
        aim_touch(w2);
        lds_barrier();
        lds_barrier();
        for (int n = 0; n <= N; ++n) {
            lds_barrier();
            if (n) store(n - 1, w2);
            lds_barrier();
            touch.chunk(N - 1 - n - kTouchAhead, s_touch[w2]);
        }
        wait_vm<0>();
        return;
    }
    if (w >= LOADS) {
        const int w2 = w - LOADS;
        LoadK lk, lk_end;
        LoadV lv, lv_end;
        const T *k = static_cast<const T *>(a.k) + q.k * DK, *qq = static_cast<const T *>(a.q) + q.k * DK;
        const T *v = static_cast<const T *>(a.dO) + q.v * d.dv + col0;
        lk.aim(rsk, w2, lane, 63);
        lv.aim(rsv, w2, lane, 63);
        lk_end.aim(rsk, w2, lane, last);
        lv_end.aim(rsv, w2, lane, last);
        auto get_k = [&](int n) { (n == 0 ? lk_end : lk).request(k + (size_t)(N - 1 - n) * 64 * rsk, s_k[n % D], w2); };
        auto get_t = [&](int n) {
            load_block<TB>(a.TT, q.blk + (N - 1 - n), s_t[n % DT], w2, lane);
            if constexpr (PRECISE) load_block<TB>(a.TT_lo, q.blk + (N - 1 - n), s_tl[n % DT], w2, lane);
        };
        auto get_q = [&](int n) {
            const int m = N - 1 - n;
            if (w2 == 0) dma16(a.coef + (q.blk + m) * kGdrCoef, lane * 16, lds_addr(s_c[n % DC]));
            (n == 0 ? lk_end : lk).request(qq + (size_t)m * 64 * rsk, s_q[n % DQ], w2);
            (n == 0 ? lv_end : lv).request(v + (size_t)m * 64 * rsv, s_do[n % DQ], w2);
        };
        if constexpr (RING) {
            // (requests of K and T^T by either wave)
            constexpr int LAST = LoadK::COUNT + (DT == D ? TB / 2048 : 0);
            reverse_ring<DT>(N, get_q, get_k, get_t, [](bool all) { all ? wait_vm<0>() : wait_vm<LAST>(); }, [] { lds_barrier(); });
        } else {
            get_q(0);
            wait_vm<0>();
            lds_barrier();
            aim_touch(w2);
            lds_barrier();
            for (int n = 0; n <= N; ++n) {
                if (n < N) {
                    get_k(n);
                    get_t(n);
                }
                if (n + 1 < N) get_q(n + 1);
                wait_vm<0>();
                lds_barrier();
                if (n) store(n - 1, w2); // (and stores, while the others multiply)
                lds_barrier();
                touch.chunk(N - 1 - n - kTouchAhead, s_touch[w2]);
                lds_barrier();
            }
            wait_vm<0>();
        }
        return;
    }

    const TileReader<T, DK> tile(r, kg);
    auto chain = [&](auto half) {
        // this wave's half (or all): of dk and of the tokens
        constexpr int TW = decltype(half)::value, HT = NT / CWS, HS = SK / CWS, H64 = S64 / CWS, RT = 4 / CWS;
        const int cg = (w - 2) / CWS, col = col0 + 16 * cg;
        int slot = 0, slot_t = 0, slot_c = 0;
        f32x4 S[HT];
        Frags<T, HT, PRECISE> Sb;
        load_state<T, TW * HT>(S, a.dS_final ? a.dS_final + q.state * DK * d.dv : nullptr, d.dv, col, r, kg);
        all_arrived();
        auto publish = [&](int n) { // D, for the storing waves and the other half's
#pragma unroll
            for (int s = 0; s < HS; ++s) {
                SlateS::put(s_s[n % CWS][cg], TW * HS + s, r, kg, Sb.hi[s]);
                if constexpr (PRECISE && CWS == 2) SlateS::put(s_sl[cg], TW * HS + s, r, kg, Sb.lo[s]);
            }
        };
        if constexpr (CWS == 2) {
            Sb.from(S);
            publish(0);
        }
        if (lane == 0) s_said[cg][TW] = 0;
        lds_barrier();
        lds_barrier();
        for (int n = 0; n <= N; ++n) {
            lds_barrier();
            if (n < N) {
                const T *k = s_k[slot], *tri = s_t[slot_t], *tri_lo = s_tl[slot_t];
                const float *c = s_c[slot_c] + G::row(0, 4 * kg);
                f32x4 X[RT], eg[4], ec[RT];
                auto decays = [&] {
#pragma unroll
                    for (int t = 0; t < 4; ++t) eg[t] = *reinterpret_cast<const f32x4 *>(c + G::row(t, 0));
#pragma unroll
                    for (int t = 0; t < RT; ++t) ec[t] = *reinterpret_cast<const f32x4 *>(c + 64 + G::row(RT * TW + t, 0));
                };
                if (RING) decays(); // (32-bit rows of 128 leave no registers for them yet)
#pragma unroll
                for (int t = 0; t < RT; ++t) X[t] = s_x[cg][RT * TW + t][lane];
                if constexpr (CWS == 1) Sb.from(S);
                const float eC = s_c[slot_c][63];
#pragma unroll
                for (int t = 0; t < HT; ++t) S[t] = eC * S[t] + s_y[cg][TW * HT + t][lane];
                lds_barrier();
                if constexpr (CWS == 1) publish(n);
                f32x4 E[RT];
                zero_acc(E);
#pragma unroll
                for (int s = 0; s < HS; ++s)
#pragma unroll
                    for (int t = 0; t < RT; ++t) E[t] = Sb.mma(tile.row_frag(k, RT * TW + t, TW * HS + s), s, E[t]);
#pragma unroll
                for (int s = (1 - TW) * HS; s < (CWS - TW) * HS; ++s) { // (no step where this wave is alone)
                    if constexpr (CWS == 2) {
                        const Frag b = SlateS::get(s_s[n % CWS][cg], s, r, kg);
                        Frag lo;
                        if constexpr (PRECISE) lo = SlateS::get(s_sl[cg], s, r, kg);
#pragma unroll
                        for (int t = 0; t < RT; ++t) {
                            const Frag f = tile.row_frag(k, RT * TW + t, s);
                            E[t] = gd_mma<T>(f, b, E[t]);
                            if constexpr (PRECISE) E[t] = gd_mma<T>(f, lo, E[t]);
                        }
                    }
                }
                if (!RING) { // (fenced in: phases mixed by the compiler need more registers than there are)
                    __builtin_amdgcn_sched_barrier(0);
                    decays();
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int t = 0; t < RT; ++t) E[t] = X[t] + ec[t] * E[t];
                Frags<T, RT, PRECISE> Eb;
                Eb.from(E);
                if constexpr (CWS == 2) {
#pragma unroll
                    for (int s = 0; s < H64; ++s) {
                        s_e[cg][TW * H64 + s][lane] = Eb.hi[s];
                        if constexpr (PRECISE) s_el[cg][TW * H64 + s][lane] = Eb.lo[s];
                    }
                    say(&s_said[cg][TW], n);
                }
                // as in the forward scan: own tokens first; sums over either half of the tokens
                f32x4 R[4], R2[2];
                zero_acc(R);
                zero_acc(R2);
                auto add = [&](int s, Frag hi, Frag lo) {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (s >= G::first(t)) {
                            f32x4 &to = CWS == 1 || s >= H64 ? R[t] : R2[t & 1];
                            const Frag f = tri_frag(tri, G::up(t, s), lane);
                            to = gd_mma<T>(f, hi, to);
                            if constexpr (PRECISE) {
                                to = gd_mma<T>(f, lo, to);
                                to = gd_mma<T>(tri_frag(tri_lo, G::up(t, s), lane), hi, to);
                            }
                        }
                };
#pragma unroll
                for (int s = 0; s < H64; ++s) add(TW * H64 + s, Eb.hi[s], Eb.lo[PRECISE ? s : 0]);
                if constexpr (CWS == 2) {
                    wait_for(&s_said[cg][1 - TW], n);
#pragma unroll
                    for (int s = 0; s < H64; ++s) {
                        const int so = (1 - TW) * H64 + s;
                        add(so, s_e[cg][so][lane], s_el[cg][PRECISE ? so : 0][lane]);
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) R[t] += R2[t];
                }
#pragma unroll
                for (int s = TW * H64; s < (TW + 1) * H64; ++s) SlateE::put(s_r + cg * SlateE::SIZE, s, r, kg, G::frag(&R[s * G::KT]));
#pragma unroll
                for (int t = 0; t < 4; ++t) R[t] *= -eg[t];
                Frags<T, 4, PRECISE> Rb;
                Rb.from(R);
#pragma unroll
                for (int s = 0; s < S64; ++s)
#pragma unroll
                    for (int t = 0; t < HT; ++t) S[t] = Rb.mma(tile.col_frag(k, TW * HT + t, s), s, S[t]);
                if constexpr (CWS == 2) {
                    Sb.from(S);
                    publish(n + 1);
                }
                slot = next_slot<D>(slot);
                slot_t = next_slot<DT>(slot_t);
                slot_c = next_slot<DC>(slot_c);
            } else {
                lds_barrier();
            }
            if constexpr (!RING) lds_barrier();
        }
        if (a.dS0) save_state<T, TW * HT>(S, a.dS0 + q.state * DK * d.dv, d.dv, col, r, kg);
    };
    if (w >= 2) { // ---- the chain
        if (CWS == 1 || w % 2 == 0) chain(std::integral_constant<int, 0>{});
        else chain(std::integral_constant<int, CWS - 1>{});
        return;
    }

    // ---- beside the chain: X of 32 tokens, Y of half of dk, all columns.  The wave's fragments of P^T are nobody else's and come straight
    // into registers, SETS chunks ahead.
    auto beside = [&](auto first_tile) {
        constexpr int T0 = decltype(first_tile)::value, HT = NT / 2;
        struct Set { Frag p[2][S64], lo[2][PRECISE ? S64 : 1]; } sets[SETS];
        int slot = 0, slot_c = 0;
        auto fetch = [&](Set &x, int n) {
            n = min(n, N - 1); // (asked for again behind the last chunk: no branch around loads in flight)
            const size_t at = (q.blk + (N - 1 - n)) * (G::NF * 64) + lane;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int s = 0; s < S64; ++s)
                    if (s >= G::first(T0 + t)) {
                        x.p[t][s] = static_cast<const Frag *>(a.PT)[at + G::up(T0 + t, s) * 64];
                        if constexpr (PRECISE) x.lo[t][s] = static_cast<const Frag *>(a.PT_lo)[at + G::up(T0 + t, s) * 64];
                    }
        };
        auto ahead = [&](Set &x, int n) { // X, Y of step n
            const T *qt = s_q[slot], *dO = s_do[slot];
            const float *c = s_c[slot_c] + G::row(0, 4 * kg);
            const int rows = n == 0 ? last + 1 : 64;
            f32x4 X[NCG][2];
            Frags<T, 4, PRECISE> Vb[NCG];
#pragma unroll
            for (int g = 0; g < NCG; ++g) {
                zero_acc(X[g]);
#pragma unroll
                for (int s = 0; s < S64; ++s) {
                    if (s < G::first(T0)) continue;
                    const Frag b = column_frag(dO, COLS, s, kg, 16 * g, r);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        if (s >= G::first(T0 + t)) {
                            X[g][t] = gd_mma<T>(x.p[t][s], b, X[g][t]);
                            if constexpr (PRECISE) X[g][t] = gd_mma<T>(x.lo[t][s], b, X[g][t]);
                        }
                }
            }
            fetch(x, n + SETS);
#pragma unroll
            for (int g = 0; g < NCG; ++g) {
#pragma unroll
                for (int t = 0; t < 2; ++t) s_x[g][T0 + t][lane] = X[g][t] * d.scale;
                f32x4 V[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    V[t] = widen4(column4(dO + G::row(t, 0) * COLS, COLS, G::row(0, 4 * kg), 16 * g, r)) *
                           (*reinterpret_cast<const f32x4 *>(c + G::row(t, 0)) * d.scale);
                    if (rows < 64) { // (what lies behind the last row is not zero)
#pragma unroll
                        for (int i = 0; i < 4; ++i) V[t][i] = G::row(t, 4 * kg) + i < rows ? V[t][i] : 0.f;
                    }
                }
                Vb[g].from(V);
            }
            f32x4 Y[NCG][HT];
#pragma unroll
            for (int g = 0; g < NCG; ++g) zero_acc(Y[g]);
#pragma unroll
            for (int s = 0; s < S64; ++s)
#pragma unroll
                for (int t = 0; t < HT; ++t) {
                    const Frag f = tile.col_frag(qt, T0 / 2 * HT + t, s);
#pragma unroll
                    for (int g = 0; g < NCG; ++g) Y[g][t] = Vb[g].mma(f, s, Y[g][t]);
                }
#pragma unroll
            for (int g = 0; g < NCG; ++g)
#pragma unroll
                for (int t = 0; t < HT; ++t) s_y[g][T0 / 2 * HT + t][lane] = Y[g][t];
            slot = next_slot<DQ>(slot);
            slot_c = next_slot<DC>(slot_c);
        };
#pragma unroll
        for (int i = 0; i < SETS; ++i) fetch(sets[i], i);
        all_arrived();
        lds_barrier();
        ahead(sets[0], 0);
        lds_barrier();
        auto turn = [&](Set &x, int n) {
            lds_barrier();
            lds_barrier();
            ahead(x, n + 1);
            if constexpr (!RING) lds_barrier();
        };
        // step 0
        lds_barrier();
        lds_barrier();
        if (N > 1) ahead(sets[SETS - 1], 1);
        if constexpr (!RING) lds_barrier();
        // steps 1 .. N - 2, whole turns without a branch inside (the compiler counts the loads in flight): X, Y of steps 2 .. N - 1
        int n = 1;
        for (; n + SETS <= N - 1; n += SETS)
#pragma unroll
            for (int i = 0; i < SETS; ++i) turn(sets[i], n + i);
        if (n <= N - 2) turn(sets[0], n++);
        // the last two steps: nothing is ahead of them
        for (; n <= N; ++n) {
            lds_barrier();
            lds_barrier();
            if constexpr (!RING) lds_barrier();
        }
    };
    if (w == 0) beside(std::integral_constant<int, 0>{});
    else beside(std::integral_constant<int, 2>{});
}

template <typename T, int DK, int NCG, bool PRECISE> hipError_t launch_cols(const GdrDims &d, const GdrScanBwdArgs &a, hipStream_t s) {
    return launch_in_parts((d.B * d.H + 7) / 8 * 8 * (d.dv / (16 * NCG)), [&](int first, dim3 grid) {
        hipLaunchKernelGGL((gdr_scan_bwd_kernel<T, DK, NCG, PRECISE>), grid, dim3((bwd_waves<T, DK, NCG, PRECISE>() * 64)), 0, s, d, a, first);
    });
}
template <typename T, int DK, bool PRECISE> hipError_t launch(const GdrDims &d, const GdrScanBwdArgs &a, hipStream_t s) {
    return gdr_one_group(d) ? launch_cols<T, DK, 1, PRECISE>(d, a, s) : launch_cols<T, DK, 2, PRECISE>(d, a, s);
}

} // namespace

hipError_t launch_gdr_scan_bwd(const GdrDims &d, const GdrScanBwdArgs &a, bool precise, hipStream_t s) {
    if (d.dtype == 1) return d.dk == 64 ? launch<float, 64, false>(d, a, s) : launch<float, 128, false>(d, a, s);
    if (precise) return d.dk == 64 ? launch<bf16_t, 64, true>(d, a, s) : launch<bf16_t, 128, true>(d, a, s);
    return d.dk == 64 ? launch<bf16_t, 64, false>(d, a, s) : launch<bf16_t, 128, false>(d, a, s);
}

} // namespace mdn
