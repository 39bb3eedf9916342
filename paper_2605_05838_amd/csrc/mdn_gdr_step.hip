// Gated delta rule, token by token (decoding):
//     S <- e^{g} S;   e = v - S^T k;   S <- S + beta k e^T;   o = scale S^T q
// Bound by reading and writing the fp32 state once per call (256 sequences of 16 heads of 128 among other work: 100 us, 5.4 TB/s; one: 2.9).  A workgroup owns COLS columns of one (sequence, value head); a thread has
// dk COLS / 1024 rows of 4 neighbouring columns in registers, so that a wave moves whole 128-byte lines; the two sums over dk go over the
// lanes of a wave, then over the four waves through LDS.  A token's operands are requested one token ahead.
#include "mdn_gdr.h"

namespace mdn {

namespace {

template <typename T, int ROWS> struct StepOps { // one token's operands of a thread, in storage form
    struct alignas(ROWS * sizeof(T)) Rows { T e[ROWS]; };
    Rows k, q;
    typename Raw4<T>::type v;
    float g, be;
};

template <typename T, int DK, int COLS, bool NT> __global__ __launch_bounds__(kThreads) void gdr_step_kernel(GdrDims d, GdrStepArgs a, int first) {
    constexpr int CG = COLS / 4, ROWS = DK * CG / kThreads; // column groups, rows of a thread
    static_assert(ROWS >= 1 && (CG == 8 || CG == 16), "lanes of a sum");
    typedef StepOps<T, ROWS> Ops;
    __shared__ __align__(16) f32x4 s_e[4][CG], s_o[4][CG];
    const int nb = d.dv / COLS, id = first + (int)blockIdx.x, bh = id / nb, b = bh / d.H, h = bh % d.H, hk = h / (d.H / d.Hk);
    const int cg = threadIdx.x % CG, sl = threadIdx.x / CG, w = wave_id();
    const int j = id % nb * COLS + cg * 4, r0 = sl * ROWS;
    auto fetch = [&](int t) {
        Ops c;
        const size_t tok = (size_t)b * d.T + t, gv = tok * d.H + h, gk = (tok * d.Hk + hk) * DK + r0;
        c.k = *reinterpret_cast<const typename Ops::Rows *>(static_cast<const T *>(a.k) + gk);
        c.q = *reinterpret_cast<const typename Ops::Rows *>(static_cast<const T *>(a.q) + gk);
        c.v = load4_raw(static_cast<const T *>(a.v) + gv * d.dv + j);
        c.g = a.g[gv];
        c.be = a.beta[gv];
        return c;
    };
    auto sum = [&](f32x4 v) { // over the rows of a wave
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (CG == 8) v[x] += dpp_move<0x128>(v[x]); // lane ^ 8
            v[x] = add_xor32(add_xor16(v[x]));
        }
        return v;
    };
    Ops c = fetch(0);
    f32x4 S[ROWS];
    f32x4 *Sg = reinterpret_cast<f32x4 *>(a.S + ((size_t)bh * DK + r0) * d.dv + j);
    const size_t ld = d.dv / 4;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) S[i] = NT ? __builtin_nontemporal_load(Sg + i * ld) : Sg[i * ld];
    for (int t = 0; t < d.T; ++t) {
        const Ops nx = fetch(t + 1 < d.T ? t + 1 : t);
        const float al = __builtin_amdgcn_exp2f(c.g * 1.44269504f);
        f32x4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            S[i] *= al;
            part += to_f32(c.k.e[i]) * S[i];
        }
        part = sum(part);
        if ((threadIdx.x & 63) < CG) s_e[w][cg] = part;
        lds_barrier();
        f32x4 e = widen4(c.v) - ((s_e[0][cg] + s_e[1][cg]) + (s_e[2][cg] + s_e[3][cg]));
        e *= c.be;
        f32x4 po = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            S[i] += to_f32(c.k.e[i]) * e;
            po += to_f32(c.q.e[i]) * S[i];
        }
        po = sum(po);
        if ((threadIdx.x & 63) < CG) s_o[w][cg] = po;
        lds_barrier();
        if (sl == 0) {
            const f32x4 o = (s_o[0][cg] + s_o[1][cg]) + (s_o[2][cg] + s_o[3][cg]);
            store4(static_cast<T *>(a.o) + (((size_t)b * d.T + t) * d.H + h) * d.dv + j, d.scale * o);
        }
        c = nx;
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (NT) __builtin_nontemporal_store(S[i], Sg + i * ld);
        else Sg[i * ld] = S[i];
    }
}

template <typename T, int DK, int COLS, bool NT> hipError_t launch_cols(const GdrDims &d, const GdrStepArgs &a, hipStream_t s) {
    return launch_in_parts(d.B * d.H * (d.dv / COLS), [&](int first, dim3 grid) {
        hipLaunchKernelGGL((gdr_step_kernel<T, DK, COLS, NT>), grid, dim3(kThreads), 0, s, d, a, first);
    });
}
// 32 columns where workgroups of 64 would leave half of the CUs without one: calls on the same states in us, 32 / 64 columns, 1 sequence of 16
// heads of 128 2.9 / 3.2, 8 4.5 / 4.5, 24 8.1 / 7.6, 256 79 / 76; 12 x 5 tokens, 8 heads of 64 x 128 in fp32 6.6 / 6.3.  States past what the
// last-level cache gives back to the next call go by it, plain / non-temporal: 256 sequences 76 / 90, 300 95 / 107, 360 130 / 128, 512 201 / 184.
template <typename T, int DK> hipError_t launch_t(const GdrDims &d, const GdrStepArgs &a, hipStream_t s) {
    const long long bytes = 4LL * d.B * d.H * DK * d.dv;
    if (2LL * d.B * d.H * (d.dv / 64) < num_cus()) return launch_cols<T, DK, 32, false>(d, a, s);
    if (bytes <= (352LL << 20)) return launch_cols<T, DK, 64, false>(d, a, s);
    return launch_cols<T, DK, 64, true>(d, a, s);
}

} // namespace

hipError_t launch_gdr_step(const GdrDims &d, const GdrStepArgs &a, hipStream_t s) {
    if (d.dtype == 1) return d.dk == 64 ? launch_t<float, 64>(d, a, s) : launch_t<float, 128>(d, a, s);
    return d.dk == 64 ? launch_t<bf16_t, 64>(d, a, s) : launch_t<bf16_t, 128>(d, a, s);
}

} // namespace mdn
