// Gated delta rule, forward scan and reconstruction of the chunk-start states.  Per chunk, S the state at its start:
//     chain:   E = T (V - e^G K S),   S <- e^{G_C} S + K^T (e^{G_C - G} beta E)
//     beside it, one chunk behind:   O = scale (e^G Q S + P E)
//     stores of E and S one chunk behind the chain, of O two
// S, E and O pass from wave to wave through LDS, rounded to the storage type.
// Bounds: HBM where all CUs have a workgroup (4 x 4 096 tokens, 16 heads, d = 128, with kept states: 520 MB in 153 us, 3.4 TB/s).  Below, the
// chain (2 050 clocks a step, 3 650 with remainders) and the CU's loads: 16 KB each of K and Q, 6 of T and P, 1 KB of V per 8 columns a step,
// of which a CU takes 25 to 37 B a clock out of the L2 (32 768 tokens: 1.45 us a step with kept states).
// PRECISE (a call that asks for the final states, which are 32-bit): S, T, V - e^G K S and e^{G_C - G} beta E enter their products as value +
// remainder (K is exact in 16 bits), so that a state carries errors of 2^-17 and not of 2^-9.
#include "mdn_gdr_scan.h"

namespace mdn {

namespace {

// Waves to 16 columns of the chain.  Two share the products, and pay for it by what they hand to each other and wait for: 48 us for 65 in
// fp32 ([2, 1 024] tokens, 4 heads, d = 64), 27 for 30 with remainders (777 tokens, 16 heads, d = 128), but 146 for 133 in 16 bits
// ([4, 4 096] tokens, 16 heads, d = 128), where one wave's products are done before the chunk behind them is there.
template <typename T, int NCG, bool PRECISE> constexpr int CW = sizeof(T) == 4 || (PRECISE && NCG == 1) ? 2 : 1;

// beside the chain, chain, loads, stores
template <typename T, int DK, int NCG, bool PRECISE, bool REBUILD> constexpr int fwd_waves() {
    return (REBUILD ? 0 : 2) + CW<T, NCG, PRECISE> * NCG + 2 + (gdr_ring<T, DK, NCG>() ? 2 : 0);
}

// REBUILD: E is given (in v's place), only the states are wanted.  KEEP: E or the states are.
template <typename T, int DK, int NCG, bool PRECISE, bool REBUILD, bool KEEP>
__global__ __launch_bounds__((fwd_waves<T, DK, NCG, PRECISE, REBUILD>() * 64)) void gdr_scan_fwd_kernel(GdrDims d, GdrScanFwdArgs a, int first) {
    typedef Gd<T> G;
    typedef typename G::Frag Frag;
    typedef Slate<T, DK> SlateS;
    typedef Slate<T, 64> SlateE;
    constexpr int NT = DK / 16, SK = DK / G::KS, S64 = 64 / G::KS, COLS = 16 * NCG, TRI = G::NF * 64 * G::E;
    constexpr int CWS = CW<T, NCG, PRECISE>, NS = CWS + 1; // NS: slots of S
    constexpr int CHAIN = REBUILD ? 0 : 2, LOADS = CHAIN + CWS * NCG, STORES = LOADS + 2; // first waves of each kind
    constexpr int TB = TRI * (int)sizeof(T);  // bytes of a triangle
    constexpr int LDO = 32 + G::E;            // row length of what a wave beside the chain stores: 32 tokens of all columns, whole rows
    constexpr int D = gdr_ring<T, DK, NCG>() ? 3 : 1; // ring depth; 1: loads between two barriers, not beside the products
    constexpr int DC = D + 1;                 // of the coefficients, which both kinds of waves read
    constexpr int SETS = sizeof(T) == 2 ? 2 : 1; // chunks of q and P that a wave beside the chain has asked for
    typedef GLoad<T, DK, true> LoadK;
    typedef GLoad<T, COLS, false> LoadV;
    __shared__ __align__(16) T s_k[D][64 * DK], s_v[D][64 * COLS], s_t[D][REBUILD ? 8 : TRI], s_tl[D][PRECISE ? TRI : 8];
    __shared__ __align__(16) float s_c[DC][kGdrCoef];
    // S: with two waves, read by the other one when it is new, beside the chain a step later, and written for the step after that meanwhile
    __shared__ __align__(16) T s_s[NS][NCG][SlateS::SIZE], s_sl[NCG][CWS == 2 && PRECISE ? SlateS::SIZE : 8];
    __shared__ __align__(16) Frag s_x[NCG][CWS == 2 ? S64 : 1][64], s_xl[NCG][CWS == 2 && PRECISE ? S64 : 1][64]; // V - e^G K S, from wave to wave
    __shared__ __align__(16) int s_touch[2][64];
    __shared__ int s_said[NCG][2]; // steps whose half of it is there
    __shared__ __align__(16) T s_e[2][REBUILD ? 8 : NCG * SlateE::SIZE], s_o[2][2][REBUILD ? 8 : COLS * LDO];

    const int w = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, kg = lane >> 4;
    int bh, sub;
    xcd_map(first + (int)blockIdx.x, d.dv / COLS, bh, sub);
    if (bh >= d.B * d.H) return;
    const GdrSeq q = gdr_seq(d, bh);
    const int col0 = sub * COLS, N = q.n, last = (q.len - 1) & 63; // last: the last row of the last chunk
    const unsigned rsv = (unsigned)(d.H * d.dv), rsk = (unsigned)(d.Hk * DK);

    // Step n: chunk n on the chain, chunk n - 1 beside it; by the two waves w2 = 0, 1 that store: S, E of chunk n - 1, O of chunk n - 2
    auto store = [&](int n, int w2) {
        // Non-temporal, but not the 32 bytes of 16 columns where later chunks are brought into the L2: these then wait there for the rest of their
        // line.  16 heads of 128 in us, non-temporal / not: 32 768 tokens 708 / 676, with kept states 868 / 829; where nothing is brought,
        // 16 384 268 / 331, and with 32 columns, 4 x 4 096, 82 / 104, the other way.
        auto tokens = [&](auto ld, void *to, int m, const T *slates, int slate_t0, int w2) {
            const size_t at = (q.v + (size_t)m * 64 * d.H) * d.dv + col0;
            const auto rows = out_rows(static_cast<T *>(to) + at, ((size_t)(m == N - 1 ? last : 63) * rsv + COLS) * sizeof(T));
            const unsigned rs = rsv * (unsigned)sizeof(T);
            const int r = lane & 15, kg = lane >> 4;
            if (sizeof(T) == 2 && NCG == 1 && a.touch) store_tokens<T, NCG, decltype(ld)::value, 0>(rows, rs, slates, slate_t0, 32 * w2, r, kg);
            else store_tokens<T, NCG, decltype(ld)::value>(rows, rs, slates, slate_t0, 32 * w2, r, kg);
        };
        if constexpr (KEEP) {
            if (n >= 1 && n <= N) {
                const int m = n - 1;
                if constexpr (!REBUILD)
                    if (a.e) tokens(std::integral_constant<int, SlateE::LD>{}, a.e, m, s_e[m & 1], 32 * w2, w2);
                if (a.states)
                    store_state<T, DK, NCG>(out_rows(static_cast<T *>(a.states) + (q.blk + m) * DK * d.dv, (size_t)DK * d.dv * sizeof(T)), s_s[m % NS], w2,
                                            col0, lane);
            }
        }
        if constexpr (!REBUILD)
            if (n >= 2) tokens(std::integral_constant<int, LDO>{}, a.o, n - 2, s_o[n & 1][w2], 0, w2);
    };
    GdrTouch<PRECISE ? 0 : touch_places((2 - REBUILD) * DK * (int)sizeof(T) + (REBUILD ? 0 : 2) * TB / 64 + 16, (int)sizeof(T), COLS)> touch;
    auto aim_touch = [&](int w2) {
        touch.aim(sub * 2 + w2, d.dv / COLS * 2, lane);
        if (!a.touch) return;
        const ptrdiff_t row = rsk * sizeof(T), rov = rsv * sizeof(T);
        touch.add(static_cast<const T *>(a.k) + q.k * DK, 64, DK * sizeof(T), row, 64 * row, N, last);
        touch.add(static_cast<const T *>(a.v) + q.v * d.dv, 64, d.dv * sizeof(T), rov, 64 * rov, N, last);
        auto block = [&](const void *t, int bytes) { touch.add(static_cast<const char *>(t) + q.blk * bytes, 1, bytes, 0, bytes, N, 0); };
        if constexpr (!REBUILD) {
            touch.add(static_cast<const T *>(a.q) + q.k * DK, 64, DK * sizeof(T), row, 64 * row, N, last);
            block(a.T, TB);
            block(a.P, TB);
        }
        block(a.coef, kGdrCoef * 4);
    };
    if (w >= STORES) {
        const int w2 = w - STORES;
        aim_touch(w2);
        for (int n = 0; n <= N + 1; ++n) {
            lds_barrier();
            store(n, w2);
            touch.chunk(n + kTouchAhead, s_touch[w2]);
        }
        wait_vm<0>();
        return;
    }
    if (w >= LOADS) {
        const int w2 = w - LOADS;
        LoadK lk, lk_end;
        LoadV lv, lv_end;
        const T *k = static_cast<const T *>(a.k) + q.k * DK, *v = static_cast<const T *>(a.v) + q.v * d.dv + col0;
        lk.aim(rsk, w2, lane, 63);
        lv.aim(rsv, w2, lane, 63);
        lk_end.aim(rsk, w2, lane, last);
        lv_end.aim(rsv, w2, lane, last);
        auto request = [&](int n) {
            if (w2 == 0) dma16(a.coef + (q.blk + n) * kGdrCoef, lane * 16, lds_addr(s_c[n % DC]));
            (n == N - 1 ? lk_end : lk).request(k + (size_t)n * 64 * rsk, s_k[n % D], w2);
            (n == N - 1 ? lv_end : lv).request(v + (size_t)n * 64 * rsv, s_v[n % D], w2);
            if constexpr (!REBUILD) load_block<TB>(a.T, q.blk + n, s_t[n % D], w2, lane);
            if constexpr (PRECISE) load_block<TB>(a.T_lo, q.blk + n, s_tl[n % D], w2, lane);
        };
        if constexpr (D == 1) {
            aim_touch(w2);
            for (int n = 0; n <= N + 1; ++n) { // (and stores, while the others multiply)
                if (n < N) request(n);
                wait_vm<0>();
                lds_barrier();
                store(n, w2);
                touch.chunk(n + kTouchAhead, s_touch[w2]);
                lds_barrier();
            }
            wait_vm<0>();
        } else {
            // requests of a chunk by either wave (the first one's coefficients included)
            constexpr int C1 = LoadK::COUNT + LoadV::COUNT + (REBUILD ? 0 : TB / 2048) + (PRECISE ? TB / 2048 : 0), C0 = C1 + 1;
            auto all_but_last = [&] { w2 == 0 ? wait_vm<C0>() : wait_vm<C1>(); };
            request(0);
            if (N > 1) {
                request(1);
                all_but_last();
            } else {
                wait_vm<0>();
            }
            for (int n = 0; n <= N + 1; ++n) {
                lds_barrier();
                if (n + 2 < N) {
                    request(n + 2);
                    all_but_last();
                } else {
                    wait_vm<0>();
                }
            }
        }
        return;
    }

    const TileReader<T, DK> tile(r, kg);
    auto chain = [&](auto half) {
        // this wave's half (or all): of dk and of the tokens
        constexpr int TW = decltype(half)::value, HT = NT / CWS, HS = SK / CWS, H64 = S64 / CWS, RT = 4 / CWS;
        const int cg = (w - CHAIN) / CWS, col = col0 + 16 * cg;
        int slot = 0, slot_c = 0, slot_s = 0;
        f32x4 S[HT];
        Frags<T, HT, PRECISE> Sb;
        load_state<T, TW * HT>(S, a.S0 ? a.S0 + q.state * DK * d.dv : nullptr, d.dv, col, r, kg);
        all_arrived();
        auto publish = [&] { // S, for the waves beside the chain and the other half's
#pragma unroll
            for (int s = 0; s < HS; ++s) {
                SlateS::put(s_s[slot_s][cg], TW * HS + s, r, kg, Sb.hi[s]);
                if constexpr (PRECISE && CWS == 2) SlateS::put(s_sl[cg], TW * HS + s, r, kg, Sb.lo[s]);
            }
        };
        // S is rounded behind the step that formed it, but by a single wave with remainders in front of the next, where the first reads take
        // their time as well: 64 us for 67 (8 x 2 048 tokens of 8 heads, d = 128); without remainders 686 for 649 (32 768 tokens of 16).
        constexpr bool BEHIND = CWS == 2 || !PRECISE;
        if (BEHIND) Sb.from(S);
        if constexpr (CWS == 2) publish();
        if (lane == 0) s_said[cg][TW] = 0;
        for (int n = 0; n <= N + 1; ++n) {
            lds_barrier();
            if (n < N) {
                const T *k = s_k[slot], *v = s_v[slot], *tri = s_t[slot], *tri_lo = s_tl[slot];
                const float *c = s_c[slot_c] + G::row(0, 4 * kg);
                const float eC = s_c[slot_c][63];
                if (!BEHIND) Sb.from(S);
                if constexpr (CWS == 1) publish();
                f32x4 E[4];
                if constexpr (REBUILD) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) E[t] = widen4(column4(v + G::row(t, 0) * COLS, COLS, G::row(0, 4 * kg), 16 * cg, r));
                } else {
                    Frag other[HS], other_lo[PRECISE ? HS : 1];
#pragma unroll
                    for (int s = 0; s < (CWS - 1) * HS; ++s) {
                        other[s] = SlateS::get(s_s[slot_s][cg], (1 - TW) * HS + s, r, kg);
                        if constexpr (PRECISE) other_lo[s] = SlateS::get(s_sl[cg], (1 - TW) * HS + s, r, kg);
                    }
                    f32x4 R[RT];
                    zero_acc(R);
#pragma unroll
                    for (int s = 0; s < HS; ++s)
#pragma unroll
                        for (int t = 0; t < RT; ++t) R[t] = Sb.mma(tile.row_frag(k, RT * TW + t, TW * HS + s), s, R[t]);
#pragma unroll
                    for (int s = 0; s < (CWS - 1) * HS; ++s)
#pragma unroll
                        for (int t = 0; t < RT; ++t) {
                            const Frag f = tile.row_frag(k, RT * TW + t, (1 - TW) * HS + s);
                            R[t] = gd_mma<T>(f, other[s], R[t]);
                            if constexpr (PRECISE) R[t] = gd_mma<T>(f, other_lo[s], R[t]);
                        }
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const int t0 = G::row(RT * TW + t, 0);
                        R[t] = widen4(column4(v + t0 * COLS, COLS, G::row(0, 4 * kg), 16 * cg, r)) - *reinterpret_cast<const f32x4 *>(c + t0) * R[t];
                    }
                    Frags<T, RT, PRECISE> Rb;
                    Rb.from(R);
                    if constexpr (CWS == 2) {
#pragma unroll
                        for (int s = 0; s < H64; ++s) {
                            s_x[cg][TW * H64 + s][lane] = Rb.hi[s];
                            if constexpr (PRECISE) s_xl[cg][TW * H64 + s][lane] = Rb.lo[s];
                        }
                        say(&s_said[cg][TW], n);
                    }
                    // Own tokens first, while the other wave's are not there yet.  Sums over either half of the tokens, so that both waves have
                    // the same bits.
                    f32x4 X[2];
                    zero_acc(E);
                    zero_acc(X);
                    auto add = [&](int s, Frag hi, Frag lo) {
#pragma unroll
                        for (int t = 0; t < 4; ++t)
                            if (s <= G::last(t)) {
                                f32x4 &to = CWS == 1 || s < H64 ? E[t] : X[t & 1];
                                const Frag f = tri_frag(tri, G::low(t, s), lane);
                                to = gd_mma<T>(f, hi, to);
                                if constexpr (PRECISE) {
                                    to = gd_mma<T>(f, lo, to);
                                    to = gd_mma<T>(tri_frag(tri_lo, G::low(t, s), lane), hi, to);
                                }
                            }
                    };
#pragma unroll
                    for (int s = 0; s < H64; ++s) add(TW * H64 + s, Rb.hi[s], Rb.lo[PRECISE ? s : 0]);
                    if constexpr (CWS == 2) {
                        wait_for(&s_said[cg][1 - TW], n);
#pragma unroll
                        for (int s = 0; s < H64; ++s) {
                            const int so = (1 - TW) * H64 + s;
                            add(so, s_x[cg][so][lane], s_xl[cg][PRECISE ? so : 0][lane]);
                        }
#pragma unroll
                        for (int t = 0; t < 2; ++t) E[2 + t] += X[t];
                    }
#pragma unroll
                    for (int s = TW * H64; s < (TW + 1) * H64; ++s) SlateE::put(s_e[n & 1] + cg * SlateE::SIZE, s, r, kg, G::frag(&E[s * G::KT]));
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) E[t] *= *reinterpret_cast<const f32x4 *>(c + 64 + G::row(t, 0));
                Frags<T, 4, PRECISE> Eb;
                Eb.from(E);
#pragma unroll
                for (int t = 0; t < HT; ++t) S[t] *= eC;
#pragma unroll
                for (int s = 0; s < S64; ++s)
#pragma unroll
                    for (int t = 0; t < HT; ++t) S[t] = Eb.mma(tile.col_frag(k, TW * HT + t, s), s, S[t]);
                slot = next_slot<D>(slot);
                slot_c = next_slot<DC>(slot_c);
                slot_s = next_slot<NS>(slot_s);
                if (BEHIND) Sb.from(S);
                if constexpr (CWS == 2) publish();
            }
            if constexpr (D == 1) lds_barrier();
        }
        if (a.S_final) save_state<T, TW * HT>(S, a.S_final + q.state * DK * d.dv, d.dv, col, r, kg);
    };
    if (w >= CHAIN) { // ---- the chain
        if (CWS == 1 || w % 2 == 0) chain(std::integral_constant<int, 0>{});
        else chain(std::integral_constant<int, CWS - 1>{});
        return;
    }

    // ---- beside the chain: 32 tokens of a chunk, all columns.  Its q rows and fragments of P are nobody else's and come straight into
    // registers, SETS chunks ahead.
    auto beside = [&](auto first_tile) {
        constexpr int T0 = decltype(first_tile)::value;
        struct Set { Frag q[2][SK], p[2][S64]; } sets[SETS];
        int slot_c = 0;
        unsigned qo[2], qo_end[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = G::row(T0 + t, r);
            qo[t] = (unsigned)row * rsk + kg * G::E;
            qo_end[t] = (unsigned)min(row, last) * rsk + kg * G::E;
        }
        auto fetch = [&](Set &x, int m) {
            m = min(m, N - 1); // (asked for again behind the last chunk: no branch around loads in flight)
            const T *qq = static_cast<const T *>(a.q) + q.k * DK + (size_t)m * 64 * rsk;
            const Frag *p = static_cast<const Frag *>(a.P) + (q.blk + m) * (G::NF * 64) + lane;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const T *row = at32(qq, m == N - 1 ? qo_end[t] : qo[t]);
#pragma unroll
                for (int s = 0; s < SK; ++s) x.q[t][s] = *reinterpret_cast<const Frag *>(row + s * G::KS);
#pragma unroll
                for (int s = 0; s < S64; ++s)
                    if (s <= G::last(T0 + t)) x.p[t][s] = p[G::low(T0 + t, s) * 64];
            }
        };
        int slot_s = 0;
        auto step = [&](Set &x, int m) {
            const T *se = s_e[m & 1];
            const float *c = s_c[slot_c] + G::row(0, 4 * kg);
            f32x4 O[NCG][2];
#pragma unroll
            for (int g = 0; g < NCG; ++g) zero_acc(O[g]);
#pragma unroll
            for (int s = 0; s < SK; ++s)
#pragma unroll
                for (int g = 0; g < NCG; ++g) {
                    const Frag b = SlateS::get(s_s[slot_s][g], s, r, kg);
#pragma unroll
                    for (int t = 0; t < 2; ++t) O[g][t] = gd_mma<T>(x.q[t][s], b, O[g][t]);
                }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int g = 0; g < NCG; ++g) O[g][t] *= *reinterpret_cast<const f32x4 *>(c + G::row(T0 + t, 0));
#pragma unroll
            for (int s = 0; s < S64; ++s)
#pragma unroll
                for (int g = 0; g < NCG; ++g) {
                    if (s > G::last(T0 + 1)) continue;
                    const Frag b = SlateE::get(se + g * SlateE::SIZE, s, r, kg);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        if (s <= G::last(T0 + t)) O[g][t] = gd_mma<T>(x.p[t][s], b, O[g][t]);
                }
            fetch(x, m + SETS);
#pragma unroll
            for (int g = 0; g < NCG; ++g) {
#pragma unroll
                for (int t = 0; t < 2; ++t) O[g][t] *= d.scale;
#pragma unroll
                for (int s = 0; s < 2 / G::KT; ++s)
                    *reinterpret_cast<Frag *>(s_o[m & 1][w] + (16 * g + r) * LDO + s * G::KS + kg * G::E) = G::frag(&O[g][s * G::KT]);
            }
            slot_c = next_slot<DC>(slot_c);
            slot_s = next_slot<NS>(slot_s);
        };
#pragma unroll
        for (int i = 0; i < SETS; ++i) fetch(sets[i], i);
        all_arrived();
        lds_barrier();
        if constexpr (D == 1) lds_barrier();
        auto turn = [&](Set &x, int m) {
            lds_barrier();
            step(x, m);
            if constexpr (D == 1) lds_barrier();
        };
        int m = 0;
        for (; m + SETS <= N; m += SETS) // (whole turns, without a branch inside: the compiler counts the loads in flight)
#pragma unroll
            for (int i = 0; i < SETS; ++i) turn(sets[i], m + i);
        if (m < N) turn(sets[0], m);
        lds_barrier();
        if constexpr (D == 1) lds_barrier();
    };
    if constexpr (!REBUILD) {
        if (w == 0) beside(std::integral_constant<int, 0>{});
        else beside(std::integral_constant<int, 2>{});
    }
}

template <typename T, int DK, int NCG, bool PRECISE, bool REBUILD, bool KEEP> hipError_t launch_keep(const GdrDims &d, const GdrScanFwdArgs &a, hipStream_t s) {
    return launch_in_parts((d.B * d.H + 7) / 8 * 8 * (d.dv / (16 * NCG)), [&](int first, dim3 grid) {
        hipLaunchKernelGGL((gdr_scan_fwd_kernel<T, DK, NCG, PRECISE, REBUILD, KEEP>), grid, dim3((fwd_waves<T, DK, NCG, PRECISE, REBUILD>() * 64)), 0, s, d, a, first);
    });
}
template <typename T, int DK, int NCG, bool PRECISE, bool REBUILD> hipError_t launch_cols(const GdrDims &d, const GdrScanFwdArgs &a, hipStream_t s) {
    if (REBUILD || a.e || a.states) return launch_keep<T, DK, NCG, PRECISE, REBUILD, true>(d, a, s);
    return launch_keep<T, DK, NCG, PRECISE, REBUILD, REBUILD>(d, a, s);
}
template <typename T, int DK, bool PRECISE, bool REBUILD> hipError_t launch(const GdrDims &d, const GdrScanFwdArgs &a, hipStream_t s) {
    return gdr_one_group(d) ? launch_cols<T, DK, 1, PRECISE, REBUILD>(d, a, s) : launch_cols<T, DK, 2, PRECISE, REBUILD>(d, a, s);
}

} // namespace

hipError_t launch_gdr_scan_fwd(const GdrDims &d, const GdrScanFwdArgs &args, bool precise, hipStream_t s) {
    GdrScanFwdArgs a = args;
    a.touch = !precise && gdr_forward_touch(d.dtype == 1, gdr_one_group(d), d.dv, args.states, gdr_call_bytes(d, 2, args.e ? 3 : 2, args.states));
    if (d.dtype == 1) return d.dk == 64 ? launch<float, 64, false, false>(d, a, s) : launch<float, 128, false, false>(d, a, s);
    if (precise) return d.dk == 64 ? launch<bf16_t, 64, true, false>(d, a, s) : launch<bf16_t, 128, true, false>(d, a, s);
    return d.dk == 64 ? launch<bf16_t, 64, false, false>(d, a, s) : launch<bf16_t, 128, false, false>(d, a, s);
}

hipError_t launch_gdr_rebuild(const GdrDims &d, const GdrScanFwdArgs &args, hipStream_t s) {
    GdrScanFwdArgs a = args;
    a.touch = d.dtype == 1 || gdr_touch_pays(gdr_call_bytes(d, 1, 1, true));
    if (d.dtype == 1) return d.dk == 64 ? launch<float, 64, false, true>(d, a, s) : launch<float, 128, false, true>(d, a, s);
    return d.dk == 64 ? launch<bf16_t, 64, false, true>(d, a, s) : launch<bf16_t, 128, false, true>(d, a, s);
}

} // namespace mdn
