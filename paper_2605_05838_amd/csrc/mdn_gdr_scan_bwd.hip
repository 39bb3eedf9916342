// Gated delta rule, reverse scan.  Per chunk, D the adjoint of the state at its END, from the last chunk to the first, dO' = scale dO:
//     beside the chain, one chunk ahead (waves 0, 1):   X = P^T dO',   Y = (e^G Q)^T dO'   (fp32, through LDS); stores of dV and D
//     chain (waves 2, 3):   dE = X + e^{G_C - G} beta K D,   dV = T^T dE,   D <- e^{G_C} D + Y - K^T (e^G dV)
// PRECISE (a call that asks for dS0, which is 32-bit): as in the forward scan; P^T and e^G dO' have remainders as well (dO and Q are exact).
#include "mdn_gdr_scan.h"

namespace mdn {

namespace {

template <typename T, int DK, bool PRECISE>
__global__ __launch_bounds__(kGdrThreads) void gdr_scan_bwd_kernel(GdrDims d, GdrScanBwdArgs a, int first) {
    typedef Gd<T> G;
    typedef GTile<T, DK> Tile;
    typedef Slate<T, DK> SlateS;
    typedef Slate<T, 64> SlateE;
    constexpr int NT = DK / 16, SK = DK / G::KS, S64 = 64 / G::KS;
    constexpr bool RING = sizeof(T) == 2; // otherwise loads between two barriers, not beside the products
    constexpr int D = RING ? 3 : 1, DQ = RING ? 2 : 1, DC = 3;
    typedef GLoad<T, DK, true> LoadK;
    typedef GLoad<T, kGdrCols, false> LoadV;
    __shared__ __align__(16) T s_k[D][64 * DK], s_q[DQ][64 * DK], s_do[DQ][64 * kGdrCols];
    __shared__ __align__(16) float s_c[DC][kGdrCoef];
    __shared__ __align__(16) f32x4 s_x[2][4][64], s_y[2][NT][64];
    __shared__ __align__(16) T s_s[2][2][SlateS::SIZE], s_r[2][2][SlateE::SIZE];

    const int w = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, kg = lane >> 4;
    int bh, sub;
    xcd_map(first + (int)blockIdx.x, d.dv / kGdrCols, bh, sub);
    if (bh >= d.B * d.H) return;
    const GdrSeq q = gdr_seq(d, bh);
    const int col0 = sub * kGdrCols, N = q.n, last = (q.len - 1) & 63; // last: the last row of the last chunk
    const unsigned rsv = (unsigned)(d.H * d.dv), rsk = (unsigned)(d.Hk * DK);

    // Step n: chunk N - 1 - n on the chain, the one before it (in time) beside it.  Barriers of a step: at its start; when the chain has
    // taken X and Y; without a ring also at its end.
    if (w >= 4) { // ---- loads
        const int w2 = w - 4;
        LoadK lk, lk_end;
        LoadV lv, lv_end;
        const T *k = static_cast<const T *>(a.k) + q.k * DK, *qq = static_cast<const T *>(a.q) + q.k * DK;
        const T *v = static_cast<const T *>(a.dO) + q.v * d.dv + col0;
        lk.aim(rsk, w2, lane, 63);
        lv.aim(rsv, w2, lane, 63);
        lk_end.aim(rsk, w2, lane, last);
        lv_end.aim(rsv, w2, lane, last);
        auto get_k = [&](int n) { (n == 0 ? lk_end : lk).request(k + (size_t)(N - 1 - n) * 64 * rsk, s_k[n % D], w2); };
        auto get_q = [&](int n) {
            (n == 0 ? lk_end : lk).request(qq + (size_t)(N - 1 - n) * 64 * rsk, s_q[n % DQ], w2);
            (n == 0 ? lv_end : lv).request(v + (size_t)(N - 1 - n) * 64 * rsv, s_do[n % DQ], w2);
            if (w2 == 0) dma16(a.coef + (q.blk + (N - 1 - n)) * kGdrCoef, lane * 16, lds_addr(s_c[n % DC]));
        };
        get_q(0);
        if constexpr (RING) {
            get_k(0);
            if (N > 1) {
                get_q(1);
                get_k(1);
            }
        }
        wait_vm<0>();
        __syncthreads();
        __syncthreads();
        for (int n = 0; n <= N; ++n) {
            if constexpr (RING) {
                __syncthreads();
                if (n + 2 < N) {
                    get_q(n + 2); // (for step n + 1)
                    get_k(n + 2);
                }
                __syncthreads();
                n + 2 < N ? wait_vm<LoadK::COUNT>() : wait_vm<0>();
            } else {
                if (n < N) get_k(n);
                if (n + 1 < N) get_q(n + 1);
                wait_vm<0>();
                __syncthreads();
                __syncthreads();
                __syncthreads();
            }
        }
        return;
    }

    const int cg = w & 1, col = col0 + 16 * cg;
    if (w >= 2) { // ---- the chain
        Triangle<T> tri;
        TriangleIf<T, PRECISE> tri_lo;
        tri.load(a.TT, q.blk + N - 1, lane);
        tri_lo.load(a.TT_lo, q.blk + N - 1, lane);
        f32x4 S[NT];
        load_state<T>(S, a.dS_final ? a.dS_final + q.state * DK * d.dv : nullptr, d.dv, col, r, kg);
        __syncthreads();
        __syncthreads();
        for (int n = 0; n <= N; ++n) {
            __syncthreads();
            if (n < N) {
                const T *k = s_k[n % D];
                const float *c = s_c[n % DC];
                f32x4 X[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) X[t] = s_x[cg][t][lane];
                Frags<T, NT, PRECISE> Sb;
                Sb.from(S);
                const float eC = c[63];
#pragma unroll
                for (int t = 0; t < NT; ++t) S[t] = eC * S[t] + s_y[cg][t][lane];
                __syncthreads();
#pragma unroll
                for (int s = 0; s < SK; ++s) SlateS::put(s_s[n & 1][cg], s, r, kg, Sb.hi[s]);
                f32x4 E[4];
                zero_acc(E);
#pragma unroll
                for (int s = 0; s < SK; ++s)
#pragma unroll
                    for (int t = 0; t < 4; ++t) E[t] = Sb.mma(Tile::row_frag(k, G::row(t, r), s, kg), s, E[t]);
#pragma unroll
                for (int t = 0; t < 4; ++t) E[t] = X[t] + *reinterpret_cast<const f32x4 *>(c + 64 + G::row(t, 4 * kg)) * E[t];
                Frags<T, 4, PRECISE> Eb;
                Eb.from(E);
                f32x4 R[4];
                zero_acc(R);
#pragma unroll
                for (int s = 0; s < S64; ++s)
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (s >= G::first(t)) {
                            R[t] = Eb.mma(tri.f[G::up(t, s)], s, R[t]);
                            if constexpr (PRECISE) R[t] = gd_mma<T>(tri_lo.f[G::up(t, s)], Eb.hi[s], R[t]);
                        }
                if (n + 1 < N) {
                    tri.load(a.TT, q.blk + N - 2 - n, lane);
                    tri_lo.load(a.TT_lo, q.blk + N - 2 - n, lane);
                }
#pragma unroll
                for (int s = 0; s < S64; ++s) SlateE::put(s_r[n & 1][cg], s, r, kg, G::frag(&R[s * G::KT]));
#pragma unroll
                for (int t = 0; t < 4; ++t) R[t] *= -*reinterpret_cast<const f32x4 *>(c + G::row(t, 4 * kg));
                Frags<T, 4, PRECISE> Rb;
                Rb.from(R);
#pragma unroll
                for (int s = 0; s < S64; ++s)
#pragma unroll
                    for (int t = 0; t < NT; ++t) S[t] = Rb.mma(Tile::col_frag(k, t, s, r, kg), s, S[t]);
            } else {
                __syncthreads();
            }
            if constexpr (!RING) __syncthreads();
        }
        if (a.dS0) save_state<T>(S, a.dS0 + q.state * DK * d.dv, d.dv, col, r, kg);
        return;
    }

    // ---- beside the chain
    Triangle<T> tri;
    TriangleIf<T, PRECISE> tri_lo;
    auto get_tri = [&](int n) {
        tri.load(a.PT, q.blk + N - 1 - n, lane);
        tri_lo.load(a.PT_lo, q.blk + N - 1 - n, lane);
    };
    if (RING) get_tri(0); // (32-bit storage: 40 registers, which are not there between the uses)
    f32x4 X[4], Y[NT];
    auto ahead = [&](int n) { // X, Y of step n
        const T *qt = s_q[n % DQ], *dO = s_do[n % DQ];
        const float *c = s_c[n % DC];
        const int rows = n == 0 ? last + 1 : 64;
        if (!RING) get_tri(n);
        zero_acc(X);
#pragma unroll
        for (int s = 0; s < S64; ++s) {
            const auto b = column_frag(dO, kGdrCols, s, kg, 16 * cg, r);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (s >= G::first(t)) {
                    X[t] = gd_mma<T>(tri.f[G::up(t, s)], b, X[t]);
                    if constexpr (PRECISE) X[t] = gd_mma<T>(tri_lo.f[G::up(t, s)], b, X[t]);
                }
        }
        if (RING && n + 1 < N) get_tri(n + 1);
        f32x4 V[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            X[t] *= d.scale;
            const int i0 = G::row(t, 4 * kg);
            V[t] = widen4(column4(dO, kGdrCols, i0, 16 * cg, r)) * (*reinterpret_cast<const f32x4 *>(c + i0) * d.scale);
#pragma unroll
            for (int x = 0; x < 4; ++x) V[t][x] = i0 + x < rows ? V[t][x] : 0.f; // (what lies behind the last row is not zero)
        }
        Frags<T, 4, PRECISE> Vb;
        Vb.from(V);
        zero_acc(Y);
#pragma unroll
        for (int s = 0; s < S64; ++s)
#pragma unroll
            for (int t = 0; t < NT; ++t) Y[t] = Vb.mma(Tile::col_frag(qt, t, s, r, kg), s, Y[t]);
    };
    auto hand_over = [&] {
#pragma unroll
        for (int t = 0; t < 4; ++t) s_x[cg][t][lane] = X[t];
#pragma unroll
        for (int t = 0; t < NT; ++t) s_y[cg][t][lane] = Y[t];
    };
    __syncthreads();
    ahead(0);
    hand_over();
    __syncthreads();
    for (int n = 0; n <= N; ++n) {
        __syncthreads();
        if (n + 1 < N) ahead(n + 1);
        __syncthreads();
        if (n + 1 < N) hand_over();
        if (n >= 1) {
            const int m = N - n, rows = n == 1 ? last + 1 : 64; // chunk of step n - 1
            store_tokens(static_cast<T *>(a.dv) + (q.v + (size_t)m * 64 * d.H) * d.dv + col, rsv, s_r[(n - 1) & 1][cg], rows, r, kg);
            store_state<T, DK>(static_cast<T *>(a.dstates) + (q.blk + m) * DK * d.dv, s_s[(n - 1) & 1][cg], cg, col0, lane);
        }
        if constexpr (!RING) __syncthreads();
    }
}

template <typename T, int DK, bool PRECISE> hipError_t launch(const GdrDims &d, const GdrScanBwdArgs &a, hipStream_t s) {
    return launch_in_parts((d.B * d.H + 7) / 8 * 8 * (d.dv / kGdrCols), [&](int first, dim3 grid) {
        hipLaunchKernelGGL((gdr_scan_bwd_kernel<T, DK, PRECISE>), grid, dim3(kGdrThreads), 0, s, d, a, first);
    });
}

} // namespace

hipError_t launch_gdr_scan_bwd(const GdrDims &d, const GdrScanBwdArgs &a, bool precise, hipStream_t s) {
    if (d.dtype == 1) return d.dk == 64 ? launch<float, 64, false>(d, a, s) : launch<float, 128, false>(d, a, s);
    if (precise) return d.dk == 64 ? launch<bf16_t, 64, true>(d, a, s) : launch<bf16_t, 128, true>(d, a, s);
    return d.dk == 64 ? launch<bf16_t, 64, false>(d, a, s) : launch<bf16_t, 128, false>(d, a, s);
}

} // namespace mdn
