// Gated delta rule, chunk-local operands: what of a 64-token chunk does not depend on the states.
//     A_ij = e^{G_i - G_j} beta_j k_i.k_j  (j < i),   P_ij = e^{G_i - G_j} beta_j q_i.k_j  (j <= i),   T = (I + A)^-1
// One workgroup of four waves per (chunk, value head).  The ten 16x16 tiles on and below the diagonal of K K^T and Q K^T are dealt
// to the waves in pairs that share a B fragment; the inverse is fp32 whatever the storage.  T, P and their transposes leave as the
// fragments that the scans load (mdn_gdr.h), triangles only: 6 KB each of 16-bit storage.  The K and Q tiles, dead after the
// products, make room for A and P: 37 KB of LDS, four workgroups per CU.  Bound by HBM where all four
// triangles are written and every value head has a key head of its own: 4 x 4 096 tokens of 16 heads of 128, 53 us for 240 MB, 4.5 TB/s.  Where
// only T and P are and heads share their keys, by what a chunk's phases wait for of each other: 16 384 tokens of 16 heads on 4 42.5 us for 86 MB, LDS
// in use 45 % of a CU's clocks, MFMA 16 %; on 16, twice the bytes, 44.0.
#include "mdn_coef.h"
#include "mdn_gdr.h"

namespace mdn {

namespace {

constexpr int LDM = 72; // row length (floats) of A and P in LDS

// the (row tile a, column tile b) pairs of wave w, three for waves 0 and 1, two for 2 and 3, as 4-bit numbers 4 a + b
constexpr unsigned kPairs[4] = {0x0dcu, 0x5feu, 0x98u, 0x4au};

template <typename T> __device__ __forceinline__ typename Gd<T>::Frag narrow(const float *x, int step, typename Gd<T>::Frag *rest) {
    f32x4 c[Gd<T>::KT];
#pragma unroll
    for (int e = 0; e < Gd<T>::E; ++e) c[e >> 2][e & 3] = x[e * step];
    const auto f = Gd<T>::frag(c);
    *rest = Gd<T>::rest(c, f);
    return f;
}

// m: 64 x 64 in LDS -> fragments of its lower triangle, or of the upper triangle of its transpose
template <typename T, bool TRANSPOSED> __device__ __forceinline__ void put_triangle(const float *m, void *to, void *to_lo, size_t blk) {
    typedef Gd<T> G;
    typedef typename G::Frag Frag;
    if (!to) return;
    Frag *hi = static_cast<Frag *>(to) + blk * (G::NF * 64), *lo = static_cast<Frag *>(to_lo) + blk * (G::NF * 64);
    for (int x = threadIdx.x; x < G::NF * 64; x += kThreads) {
        const int f = x / 64, r = x & 15, kg = x >> 4 & 3;
        int t = 0, s = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int v = 0; v < 64 / G::KS; ++v)
                if (TRANSPOSED ? v >= G::first(u) && G::up(u, v) == f : v <= G::last(u) && G::low(u, v) == f) t = u, s = v;
        const int row = G::row(t, r), k0 = s * G::KS + kg * G::E;
        Frag rest;
        const Frag v = TRANSPOSED ? narrow<T>(m + k0 * LDM + row, LDM, &rest) : narrow<T>(m + row * LDM + k0, 1, &rest);
        hi[x] = v;
        if (to_lo) lo[x] = rest;
    }
}

template <typename T, int DK> __global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 1) void gdr_local_kernel(GdrDims d, GdrLocalArgs a, int first) {
    typedef Op<T> O;
    constexpr int CPR = DK / Gd<T>::E, XM = (CPR < 16 ? CPR : 16) - 1;
    constexpr int TILES = 2 * 64 * DK * (int)sizeof(T), MATS = 2 * 64 * LDM * 4;
    __shared__ __align__(16) char s_mem[TILES > MATS ? TILES : MATS];
    __shared__ float s_hi[64], s_lo[64], s_be[64];
    T *sK = reinterpret_cast<T *>(s_mem), *sQ = sK + 64 * DK;
    float *sA = reinterpret_cast<float *>(s_mem), *sP = sA + 64 * LDM;

    const int id = first + (int)blockIdx.x, h = id % d.H, hk = h / (d.H / d.Hk);
    const GdrChunk p = gdr_chunk(d, id / d.H, h);
    const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, kg = lane >> 4;
    const size_t gate = (p.tok + min(lane, p.rows - 1)) * d.H + h;
    float g = a.g[gate], be = a.beta[gate];
    const unsigned rs = (unsigned)(d.Hk * DK);
    const size_t key = (p.tok * d.Hk + hk) * DK;
    dma_token_tile<T, DK, 4, false>(sK, static_cast<const T *>(a.k) + key, rs, w, lane, p.rows - 1);
    dma_token_tile<T, DK, 4, false>(sQ, static_cast<const T *>(a.q) + key, rs, w, lane, p.rows - 1);
    if (lane >= p.rows) g = be = 0.f;
    GdrDecay dec;
    dec.sums(g, lane);
    if (w == 0) {
        s_hi[lane] = dec.hi;
        s_lo[lane] = dec.lo;
        s_be[lane] = be;
        const float hC = lane_value(dec.hi, 63), lC = lane_value(dec.lo, 63);
        float *c = a.coef + p.blk * kGdrCoef;
        c[lane] = GdrDecay::pow2(dec.hi, dec.lo);
        c[64 + lane] = be * GdrDecay::pow2(hC - dec.hi, lC - dec.lo);
    }
    wait_vm<0>();
    lds_barrier();

    auto row_frag = [&](const T *t, int row, int st) {
        return O::load(t + row * DK + ((st * 4 + kg) ^ (row & XM)) * Gd<T>::E);
    };
    const unsigned pairs = kPairs[w];
    f32x4 kk[3], qk[3];
    zero_acc(kk);
    zero_acc(qk);
#pragma unroll
    for (int u = 0; u < 3; ++u) {
        const int ta = pairs >> (4 * u + 2) & 3, tb = pairs >> (4 * u) & 3;
        if (u < 2 || w < 2) {
#pragma unroll
            for (int st = 0; st < DK / O::KSTEP; ++st) {
                const auto b = row_frag(sK, 16 * tb + r, st);
                kk[u] = O::mma(row_frag(sK, 16 * ta + r, st), b, kk[u]);
                qk[u] = O::mma(row_frag(sQ, 16 * ta + r, st), b, qk[u]);
            }
        }
    }
    lds_barrier();
    auto put = [&](int ta, int tb, f32x4 kv, f32x4 qv) {
        const int j = 16 * tb + r;
        const float hj = s_hi[j], lj = s_lo[j], bj = s_be[j];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int i = 16 * ta + 4 * kg + x;
            const float c = bj * GdrDecay::pow2(s_hi[i] - hj, s_lo[i] - lj);
            sA[i * LDM + j] = i > j && i < p.rows ? c * kv[x] : 0.f;
            sP[i * LDM + j] = i >= j && i < p.rows ? c * qv[x] : 0.f;
        }
    };
#pragma unroll
    for (int u = 0; u < 3; ++u)
        if (u < 2 || w < 2) put(pairs >> (4 * u + 2) & 3, pairs >> (4 * u) & 3, kk[u], qk[u]);
    if (w >= 2) { // the tiles beside the diagonal that a 32-wide step of the rows above it reads
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int i = 32 * (w - 2) + 4 * kg + x, j = 32 * (w - 2) + 16 + r;
            sA[i * LDM + j] = sP[i * LDM + j] = 0.f;
        }
    }
    lds_barrier();
    tri_inverse_blocked(sA, LDM, w);
    lds_barrier();
    put_triangle<T, false>(sA, a.T, a.T_lo, p.blk);
    put_triangle<T, false>(sP, a.P, nullptr, p.blk);
    put_triangle<T, true>(sA, a.TT, a.TT_lo, p.blk);
    put_triangle<T, true>(sP, a.PT, a.PT_lo, p.blk);
}

template <typename T, int DK> hipError_t launch(const GdrDims &d, const GdrLocalArgs &a, hipStream_t s) {
    return launch_in_parts(d.nchunks * d.H, [&](int first, dim3 grid) {
        hipLaunchKernelGGL((gdr_local_kernel<T, DK>), grid, dim3(kThreads), 0, s, d, a, first);
    });
}

} // namespace

hipError_t launch_gdr_local(const GdrDims &d, const GdrLocalArgs &a, hipStream_t s) {
    if (d.dtype == 1) return d.dk == 64 ? launch<float, 64>(d, a, s) : launch<float, 128>(d, a, s);
    return d.dk == 64 ? launch<bf16_t, 64>(d, a, s) : launch<bf16_t, 128>(d, a, s);
}

} // namespace mdn
