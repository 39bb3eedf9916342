// Gated delta rule, forward scan and reconstruction of the chunk-start states.  Per chunk, S the state at its start:
//     chain (waves 2, 3):   E = T (V - e^G K S),   S <- e^{G_C} S + K^T (e^{G_C - G} beta E)
//     beside it, one chunk behind (waves 0, 1):   O = scale (e^G Q S + P E); stores of O, E and S
// S and E reach the waves beside the chain through LDS, rounded to the storage type.
// Bounds: a chunk's tiles are read by dv / 32 workgroups, of one XCD: 48 KB a step and CU at d = 128, which out of HBM and L2 arrive at
// 37 B a clock and CU (1 320 clocks); the chain has 38 products of 16x16x32 (PRECISE 82) of 16 clocks on its SIMD.
// PRECISE (a call that asks for the final states, which are 32-bit): S, T, V - e^G K S and e^{G_C - G} beta E enter their products as value +
// remainder (K is exact in 16 bits), so that a state carries errors of 2^-17 and not of 2^-9.
#include "mdn_gdr_scan.h"

namespace mdn {

namespace {

// REBUILD: E is given (in v's place), only the states are wanted
template <typename T, int DK, bool PRECISE, bool REBUILD>
__global__ __launch_bounds__(kGdrThreads) void gdr_scan_fwd_kernel(GdrDims d, GdrScanFwdArgs a, int first) {
    typedef Gd<T> G;
    typedef GTile<T, DK> Tile;
    typedef Slate<T, DK> SlateS;
    typedef Slate<T, 64> SlateE;
    constexpr int NT = DK / 16, SK = DK / G::KS, S64 = 64 / G::KS;
    constexpr int D = sizeof(T) == 2 ? 3 : 1; // ring depth; 1: loads between two barriers, not beside the products
    constexpr int DC = D + 1;                 // of the coefficients, which both kinds of waves read
    typedef GLoad<T, DK, true> LoadK;
    typedef GLoad<T, kGdrCols, false> LoadV;
    __shared__ __align__(16) T s_k[D][64 * DK], s_q[D][REBUILD ? 8 : 64 * DK], s_v[D][64 * kGdrCols];
    __shared__ __align__(16) float s_c[DC][kGdrCoef];
    __shared__ __align__(16) T s_s[2][2][SlateS::SIZE], s_e[2][2][REBUILD ? 8 : SlateE::SIZE], s_o[2][REBUILD ? 8 : SlateE::SIZE];

    const int w = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, kg = lane >> 4;
    int bh, sub;
    xcd_map(first + (int)blockIdx.x, d.dv / kGdrCols, bh, sub);
    if (bh >= d.B * d.H) return;
    const GdrSeq q = gdr_seq(d, bh);
    const int col0 = sub * kGdrCols, N = q.n, last = (q.len - 1) & 63; // last: the last row of the last chunk
    const unsigned rsv = (unsigned)(d.H * d.dv), rsk = (unsigned)(d.Hk * DK);

    // Step n: chunk n on the chain, chunk n - 1 beside it
    if (w >= 4) { // ---- loads
        const int w2 = w - 4;
        LoadK lk, lk_end;
        LoadV lv, lv_end;
        const T *k = static_cast<const T *>(a.k) + q.k * DK, *qq = static_cast<const T *>(a.q) + q.k * DK;
        const T *v = static_cast<const T *>(a.v) + q.v * d.dv + col0;
        lk.aim(rsk, w2, lane, 63);
        lv.aim(rsv, w2, lane, 63);
        lk_end.aim(rsk, w2, lane, last);
        lv_end.aim(rsv, w2, lane, last);
        auto get_kv = [&](int n) {
            (n == N - 1 ? lk_end : lk).request(k + (size_t)n * 64 * rsk, s_k[n % D], w2);
            (n == N - 1 ? lv_end : lv).request(v + (size_t)n * 64 * rsv, s_v[n % D], w2);
            if (w2 == 0) dma16(a.coef + (q.blk + n) * kGdrCoef, lane * 16, lds_addr(s_c[n % DC]));
        };
        auto get_q = [&](int n) {
            if constexpr (!REBUILD) (n == N - 1 ? lk_end : lk).request(qq + (size_t)n * 64 * rsk, s_q[n % D], w2);
        };
        if constexpr (D == 1) {
            for (int n = 0; n <= N; ++n) {
                if (n >= 1) get_q(n - 1);
                if (n < N) get_kv(n);
                wait_vm<0>();
                __syncthreads();
                __syncthreads();
            }
        } else {
            constexpr int KV = LoadK::COUNT + LoadV::COUNT, STEP = KV + (REBUILD ? 0 : LoadK::COUNT);
            get_kv(0);
            get_q(0);
            if (N > 1) {
                get_kv(1);
                w2 == 0 ? wait_vm<KV + 1>() : wait_vm<KV>();
            } else {
                wait_vm<0>();
            }
            for (int n = 0; n <= N; ++n) {
                __syncthreads();
                if (n + 1 < N) get_q(n + 1); // (for step n + 2)
                if (n + 2 < N) {
                    get_kv(n + 2);
                    w2 == 0 ? wait_vm<STEP + 1>() : wait_vm<STEP>();
                } else {
                    wait_vm<0>();
                }
            }
        }
        return;
    }

    const int cg = w & 1, col = col0 + 16 * cg;
    if (w >= 2) { // ---- the chain
        Triangle<T> tri;
        TriangleIf<T, PRECISE> tri_lo;
        if constexpr (!REBUILD) {
            tri.load(a.T, q.blk, lane);
            tri_lo.load(a.T_lo, q.blk, lane);
        }
        f32x4 S[NT];
        load_state<T>(S, a.S0 ? a.S0 + q.state * DK * d.dv : nullptr, d.dv, col, r, kg);
        for (int n = 0; n <= N; ++n) {
            __syncthreads();
            if (n < N) {
                const T *k = s_k[n % D], *v = s_v[n % D];
                const float *c = s_c[n % DC];
                Frags<T, NT, PRECISE> Sb;
                Sb.from(S);
#pragma unroll
                for (int s = 0; s < SK; ++s) SlateS::put(s_s[n & 1][cg], s, r, kg, Sb.hi[s]);
                f32x4 E[4];
                if constexpr (REBUILD) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) E[t] = widen4(column4(v, kGdrCols, G::row(t, 4 * kg), 16 * cg, r));
                } else {
                    f32x4 R[4];
                    zero_acc(R);
#pragma unroll
                    for (int s = 0; s < SK; ++s)
#pragma unroll
                        for (int t = 0; t < 4; ++t) R[t] = Sb.mma(Tile::row_frag(k, G::row(t, r), s, kg), s, R[t]);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const f32x4 eg = *reinterpret_cast<const f32x4 *>(c + G::row(t, 4 * kg));
                        R[t] = widen4(column4(v, kGdrCols, G::row(t, 4 * kg), 16 * cg, r)) - eg * R[t];
                    }
                    Frags<T, 4, PRECISE> Rb;
                    Rb.from(R);
                    zero_acc(E);
#pragma unroll
                    for (int s = 0; s < S64; ++s)
#pragma unroll
                        for (int t = 0; t < 4; ++t)
                            if (s <= G::last(t)) {
                                E[t] = Rb.mma(tri.f[G::low(t, s)], s, E[t]);
                                if constexpr (PRECISE) E[t] = gd_mma<T>(tri_lo.f[G::low(t, s)], Rb.hi[s], E[t]);
                            }
                    if (n + 1 < N) {
                        tri.load(a.T, q.blk + n + 1, lane);
                        tri_lo.load(a.T_lo, q.blk + n + 1, lane);
                    }
#pragma unroll
                    for (int s = 0; s < S64; ++s) SlateE::put(s_e[n & 1][cg], s, r, kg, G::frag(&E[s * G::KT]));
                }
                const float eC = c[63];
#pragma unroll
                for (int t = 0; t < 4; ++t) E[t] *= *reinterpret_cast<const f32x4 *>(c + 64 + G::row(t, 4 * kg));
                Frags<T, 4, PRECISE> Eb;
                Eb.from(E);
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t] *= eC;
#pragma unroll
                for (int s = 0; s < S64; ++s)
#pragma unroll
                    for (int t = 0; t < NT; ++t) S[t] = Eb.mma(Tile::col_frag(k, t, s, r, kg), s, S[t]);
            }
            if constexpr (D == 1) __syncthreads();
        }
        if (a.S_final) save_state<T>(S, a.S_final + q.state * DK * d.dv, d.dv, col, r, kg);
        return;
    }

    // ---- beside the chain
    Triangle<T> tri;
    if constexpr (!REBUILD) tri.load(a.P, q.blk, lane);
    for (int n = 0; n <= N; ++n) {
        __syncthreads();
        if (n >= 1) {
            const int m = n - 1, rows = m == N - 1 ? last + 1 : 64;
            const T *ss = s_s[m & 1][cg];
            if constexpr (!REBUILD) {
                const T *qt = s_q[m % D], *se = s_e[m & 1][cg];
                const float *c = s_c[m % DC];
                f32x4 O[4];
                zero_acc(O);
#pragma unroll
                for (int s = 0; s < SK; ++s) {
                    const auto b = SlateS::get(ss, s, r, kg);
#pragma unroll
                    for (int t = 0; t < 4; ++t) O[t] = gd_mma<T>(Tile::row_frag(qt, G::row(t, r), s, kg), b, O[t]);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) O[t] *= *reinterpret_cast<const f32x4 *>(c + G::row(t, 4 * kg));
#pragma unroll
                for (int s = 0; s < S64; ++s) {
                    const auto b = SlateE::get(se, s, r, kg);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (s <= G::last(t)) O[t] = gd_mma<T>(tri.f[G::low(t, s)], b, O[t]);
                }
                if (n < N) tri.load(a.P, q.blk + n, lane);
#pragma unroll
                for (int t = 0; t < 4; ++t) O[t] *= d.scale;
#pragma unroll
                for (int s = 0; s < S64; ++s) SlateE::put(s_o[cg], s, r, kg, G::frag(&O[s * G::KT]));
                const size_t at = (q.v + (size_t)m * 64 * d.H) * d.dv + col;
                store_tokens(static_cast<T *>(a.o) + at, rsv, s_o[cg], rows, r, kg);
                if (a.e) store_tokens(static_cast<T *>(a.e) + at, rsv, se, rows, r, kg);
            }
            if (a.states) store_state<T, DK>(static_cast<T *>(a.states) + (q.blk + m) * DK * d.dv, ss, cg, col0, lane);
        }
        if constexpr (D == 1) __syncthreads();
    }
}

template <typename T, int DK, bool PRECISE, bool REBUILD> hipError_t launch(const GdrDims &d, const GdrScanFwdArgs &a, hipStream_t s) {
    return launch_in_parts((d.B * d.H + 7) / 8 * 8 * (d.dv / kGdrCols), [&](int first, dim3 grid) {
        hipLaunchKernelGGL((gdr_scan_fwd_kernel<T, DK, PRECISE, REBUILD>), grid, dim3(kGdrThreads), 0, s, d, a, first);
    });
}

} // namespace

hipError_t launch_gdr_scan_fwd(const GdrDims &d, const GdrScanFwdArgs &a, bool precise, hipStream_t s) {
    if (d.dtype == 1) return d.dk == 64 ? launch<float, 64, false, false>(d, a, s) : launch<float, 128, false, false>(d, a, s);
    if (precise) return d.dk == 64 ? launch<bf16_t, 64, true, false>(d, a, s) : launch<bf16_t, 128, true, false>(d, a, s);
    return d.dk == 64 ? launch<bf16_t, 64, false, false>(d, a, s) : launch<bf16_t, 128, false, false>(d, a, s);
}

hipError_t launch_gdr_rebuild(const GdrDims &d, const GdrScanFwdArgs &a, hipStream_t s) {
    if (d.dtype == 1) return d.dk == 64 ? launch<float, 64, false, true>(d, a, s) : launch<float, 128, false, true>(d, a, s);
    return d.dk == 64 ? launch<bf16_t, 64, false, true>(d, a, s) : launch<bf16_t, 128, false, true>(d, a, s);
}

} // namespace mdn
