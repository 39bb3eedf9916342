// 8-bit checkpoints of the rows that the layer's elementwise operations need again in the backward, and those operations from them.
// A row of [B,T,H,d] is kept as blocks of 32 values: one exponent byte e (step 2^(e - 127)) and 32 signed codes,
//     step = 2^(floor(log2 max|x|) - 6),   code = round(x / step) to the nearest even, at most 127 in size,   x ~ code * step:
// 1 + 1/32 bytes a value where 16-bit storage takes 2.  Steps are powers of two, so that nothing but the one rounding of a code (half a
// step, 2^-7 of the block's largest value) is lost and every value is exact in either storage type.  A block with an infinity or a NaN keeps e = 255 and codes
// of 0: 0 * 2^128 reads back as NaN.
// Streaming kernels like those of mdn_layer_ops.hip, with the checkpoint written in the pass that reads the row anyway.  A lane has 8 (or 4) values;
// the largest of 32 goes over 4 (or 8) lanes.  Parameter gradients are summed in a fixed order: dw in each lane, then over the lanes,
// waves and workgroups one after the other; dd as a value per row, then over slabs of tokens.
// Bound by HBM, 4 x 4 096 tokens of 16 heads of 128 in 16 bits: front end with checkpoints 98 us (5.1 TB/s), from them 69 (4.4), its backward 106
// (4.8); back end with checkpoints 56 (4.8), its backward 64 (4.2); one tensor's checkpoint by itself 18, read back 16 (out of the last-level cache in part).
#include "mdn_kept_rules.h"
#include "mdn_layer_rows.h"

namespace mdn {

namespace {

// E values of a lane out of a block of 32, as codes
template <int E> struct Codes {
    static_assert(E == 8 || E == 4, "16 bytes of storage");
    typedef typename std::conditional<E == 8, uint64_t, uint32_t>::type __attribute__((aligned(1))) Word;
    static __device__ __forceinline__ int block_max(int x) { // over the lanes of a block
        auto step = [&](int y) { x = x > y ? x : y; };
        step(__builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, true));  // quad_perm [1,0,3,2]
        step(__builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, true));  // quad_perm [2,3,0,1]
        if (E == 4) step(__builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true)); // row_half_mirror
        return x;
    }
    static __device__ __forceinline__ void keep(const float (&v)[E], int8_t *codes, uint8_t *exponents, size_t at) {
        int top = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int b = __float_as_int(v[e]) & 0x7fffffff; // (as integers: an infinity is above every number, a NaN above that)
            top = top > b ? top : b;
        }
        top = block_max(top);
        const int biased = (top >> 23) - 6, ex = top >= 0x7f800000 ? 255 : biased > 1 ? biased : 1;
        const float inv = ex == 255 ? 0.f : __int_as_float((254 - ex) << 23);
        Word w = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            int c = (int)__builtin_rintf(ex == 255 ? 0.f : v[e] * inv);
            c = c > 127 ? 127 : c < -127 ? -127 : c;
            w |= (Word)(uint8_t)c << (8 * e);
        }
        __builtin_nontemporal_store(w, reinterpret_cast<Word *>(codes + at));
        if (at % 32 == 0) exponents[at / 32] = (uint8_t)ex;
    }
    static __device__ __forceinline__ void load(float (&v)[E], const int8_t *codes, const uint8_t *exponents, size_t at) {
        const Word w = *reinterpret_cast<const Word *>(codes + at);
        const float step = __int_as_float((int)exponents[at / 32] << 23);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (float)(int8_t)(w >> (8 * e)) * step;
    }
};

struct Kept {
    int8_t *codes;
    uint8_t *exponents;
};
template <int N> struct KeptSet { Kept t[N]; };

template <typename T, int D> struct Rows : Row<T, D, 16 / (int)sizeof(T)> {
    static constexpr int E = 16 / (int)sizeof(T);
    __device__ __forceinline__ void keep(const Kept &k, size_t at) const { Codes<E>::keep(this->v, k.codes, k.exponents, at); }
    __device__ __forceinline__ void recall(const Kept &k, size_t at) { Codes<E>::load(this->v, k.codes, k.exponents, at); }
};

// x -> kept (PACK) or kept -> x
template <typename T, int D, bool PACK> __global__ __launch_bounds__(LT) void kept_copy_kernel(LayerDims d, T *x, Kept k) {
    typedef Rows<T, D> R;
    for (RowWalk w(d, R::RPW, R::LPR); w.row < d.rows; w.next(d)) {
        const size_t o = (size_t)w.row * D + (lane_id() % R::LPR) * R::E;
        R a;
        if (PACK) {
            a.load(x + o);
            a.keep(k, o);
        } else {
            a.recall(k, o);
            a.store(x + o);
        }
    }
}

// FROM_KEPT: the inputs are checkpoints; otherwise they are rows, of which checkpoints are written
template <typename T, int D, bool FROM_KEPT>
__global__ __launch_bounds__(LT) void frontend_fwd_kept_kernel(LayerDims d, const T *xq, const T *xk, const T *xv, KeptSet<3> kept, const float *dh,
                                                                float eps, T *q, T *k, T *v) {
    typedef Rows<T, D> R;
    for (RowWalk w(d, R::RPW, R::LPR); w.row < d.rows; w.next(d)) {
        const size_t o = (size_t)w.row * D + (lane_id() % R::LPR) * R::E;
        R a, b, c;
        if (FROM_KEPT) {
            a.recall(kept.t[0], o);
            b.recall(kept.t[1], o);
            c.recall(kept.t[2], o);
        } else {
            a.load(xq + o);
            b.load(xk + o);
            c.load(xv + o);
            a.keep(kept.t[0], o);
            b.keep(kept.t[1], o);
            c.keep(kept.t[2], o);
        }
        const float dc = dh[w.h];
        float sq = 0.f, sk = 0.f;
#pragma unroll
        for (int e = 0; e < R::E; ++e) {
            b.v[e] *= sigm(b.v[e]);
            a.v[e] = a.v[e] * sigm(a.v[e]) - dc * b.v[e];
            sq += a.v[e] * a.v[e];
            sk += b.v[e] * b.v[e];
        }
        const float iq = rsqrtf(R::row_sum(sq) + eps), ik = rsqrtf(R::row_sum(sk) + eps);
#pragma unroll
        for (int e = 0; e < R::E; ++e) {
            a.v[e] *= iq;
            b.v[e] *= ik;
            c.v[e] *= sigm(c.v[e]);
        }
        a.store(q + o);
        b.store(k + o);
        c.store(v + o);
    }
}

// row_dd: a row's share of dd, or null
template <typename T, int D>
__global__ __launch_bounds__(LT) void frontend_bwd_kept_kernel(LayerDims d, KeptSet<3> kept, const float *dh, float eps, const T *dq, const T *dk,
                                                                const T *dv, T *dxq, T *dxk, T *dxv, float *row_dd) {
    typedef Rows<T, D> R;
    for (RowWalk w(d, R::RPW, R::LPR); w.row < d.rows; w.next(d)) {
        const size_t o = (size_t)w.row * D + (lane_id() % R::LPR) * R::E;
        R a, b, c, ga, gb, gc;
        a.recall(kept.t[0], o);
        b.recall(kept.t[1], o);
        ga.load(dq + o);
        gb.load(dk + o);
        c.recall(kept.t[2], o);
        gc.load(dv + o);
        const float dc = dh[w.h];
        // SiLU(x) = x s, SiLU'(x) = s (1 + x (1 - s)): the derivatives replace the inputs
        float qc[R::E], ks[R::E], sq = 0.f, sk = 0.f;
#pragma unroll
        for (int e = 0; e < R::E; ++e) {
            const float sa = sigm(a.v[e]), sb = sigm(b.v[e]);
            ks[e] = b.v[e] * sb;
            qc[e] = a.v[e] * sa - dc * ks[e];
            a.v[e] = sa * (1.f + a.v[e] * (1.f - sa));
            b.v[e] = sb * (1.f + b.v[e] * (1.f - sb));
            sq += qc[e] * qc[e];
            sk += ks[e] * ks[e];
        }
        const float iq = rsqrtf(R::row_sum(sq) + eps), ik = rsqrtf(R::row_sum(sk) + eps);
        float dotq = 0.f, dotk = 0.f;
#pragma unroll
        for (int e = 0; e < R::E; ++e) {
            qc[e] *= iq;
            dotq += qc[e] * ga.v[e];
            dotk += ks[e] * gb.v[e];
        }
        dotq = R::row_sum(dotq);
        dotk = R::row_sum(dotk) * ik * ik;
        float ddp = 0.f;
#pragma unroll
        for (int e = 0; e < R::E; ++e) {
            const float dqc = (ga.v[e] - qc[e] * dotq) * iq; // through the L2 norm of q' - d k'
            const float dks = (gb.v[e] - ks[e] * dotk) * ik - dc * dqc;
            ddp -= dqc * ks[e];
            a.v[e] *= dqc;
            b.v[e] *= dks;
            const float sc = sigm(c.v[e]);
            c.v[e] = gc.v[e] * (sc * (1.f + c.v[e] * (1.f - sc)));
        }
        a.store(dxq + o);
        b.store(dxk + o);
        c.store(dxv + o);
        if (row_dd) {
            ddp = R::row_sum(ddp);
            if (lane_id() % R::LPR == 0) row_dd[w.row] = ddp;
        }
    }
}

// from: [tokens][H] -> to: [gridDim.x][H], workgroup b the sum over its slab of tokens; one workgroup: the sum.  (Eight loads on their way at
// a time: one after the other, 777 tokens of 16 heads took a workgroup 30 us.)
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void sum_tokens_kernel(const float *from, float *to, int tokens, int H) {
    __shared__ float s[kSumThreads];
    const int per = (tokens + gridDim.x - 1) / gridDim.x, t0 = blockIdx.x * per, t1 = min(tokens, t0 + per);
    for (int h0 = 0; h0 < H; h0 += kSumThreads) {
        const int n = min(kSumThreads, H - h0), groups = kSumThreads / n, g = threadIdx.x / n, h = h0 + threadIdx.x % n; // groups of n threads take turns
        float x = 0.f;
        if (g < groups)
            for (int t = t0 + g; t < t1; t += 8 * groups) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = t + i * groups < t1 ? from[(size_t)(t + i * groups) * H + h] : 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) x += v[i];
            }
        s[threadIdx.x] = x;
        __syncthreads();
        if (g == 0) {
            for (int i = 1; i < groups; ++i) x += s[i * n + threadIdx.x];
            to[(size_t)blockIdx.x * H + h] = x;
        }
        __syncthreads();
    }
}

template <typename T, int D>
__global__ __launch_bounds__(LT) void epilogue_fwd_keep_kernel(LayerDims d, const T *o, const T *g, KeptSet<2> kept, const float *w, float eps, T *y) {
    typedef Rows<T, D> R;
    Row<float, D, R::E> wr;
    wr.load(w + (lane_id() % R::LPR) * R::E);
    for (RowWalk k(d, R::RPW, R::LPR); k.row < d.rows; k.next(d)) {
        const size_t off = (size_t)k.row * D + (lane_id() % R::LPR) * R::E;
        R a, b;
        a.load(o + off);
        b.load(g + off);
        a.keep(kept.t[0], off);
        b.keep(kept.t[1], off);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < R::E; ++e) ss += a.v[e] * a.v[e];
        const float ir = rsqrtf(R::row_sum(ss) * (1.f / D) + eps);
#pragma unroll
        for (int e = 0; e < R::E; ++e) a.v[e] = sigm(b.v[e]) * wr.v[e] * a.v[e] * ir;
        a.store(y + off);
    }
}

// part_dw: [gridDim.x][D], the workgroups' shares of dw, or null
template <typename T, int D>
__global__ __launch_bounds__(1024) void epilogue_bwd_kept_kernel(LayerDims d, KeptSet<2> kept, const float *w, float eps, const T *dy, T *dout, T *dg,
                                                                  float *part_dw) {
    typedef Rows<T, D> R;
    __shared__ float s_dw[16][D];
    const int col = (lane_id() % R::LPR) * R::E;
    Row<float, D, R::E> wr;
    wr.load(w + col);
    float dwp[R::E];
#pragma unroll
    for (int e = 0; e < R::E; ++e) dwp[e] = 0.f;
    for (RowWalk k(d, R::RPW, R::LPR); k.row < d.rows; k.next(d)) {
        const size_t off = (size_t)k.row * D + col;
        R a, b, c;
        a.recall(kept.t[0], off);
        b.recall(kept.t[1], off);
        c.load(dy + off);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < R::E; ++e) ss += a.v[e] * a.v[e];
        const float ir = rsqrtf(R::row_sum(ss) * (1.f / D) + eps);
        float dn[R::E], dot = 0.f;
#pragma unroll
        for (int e = 0; e < R::E; ++e) {
            const float sg = sigm(b.v[e]), t = c.v[e] * sg;
            a.v[e] *= ir; // normalised output
            dn[e] = t * wr.v[e];
            dot += a.v[e] * dn[e];
            dwp[e] += t * a.v[e];
            b.v[e] = dn[e] * a.v[e] * (1.f - sg);
        }
        dot = R::row_sum(dot) * (1.f / D);
#pragma unroll
        for (int e = 0; e < R::E; ++e) a.v[e] = (dn[e] - a.v[e] * dot) * ir;
        a.store(dout + off);
        b.store(dg + off);
    }
    if (part_dw) {
        // the rows of a wave first (lanes with the same columns), then the waves one after the other
#pragma unroll
        for (int e = 0; e < R::E; ++e) {
            if (R::LPR == 8) dwp[e] += dpp_move<0x128>(dwp[e]); // row_ror 8
            if (R::LPR <= 16) dwp[e] = add_xor16(dwp[e]);
            if (R::LPR <= 32) dwp[e] = add_xor32(dwp[e]);
            if (lane_id() < R::LPR) s_dw[wave_id()][col + e] = dwp[e];
        }
        __syncthreads();
        const int waves = blockDim.x >> 6;
        for (int c = threadIdx.x; c < D; c += blockDim.x) {
            float x = s_dw[0][c];
            for (int i = 1; i < waves; ++i) x += s_dw[i][c];
            part_dw[(size_t)blockIdx.x * D + c] = x;
        }
    }
}

int status() { return hipGetLastError() == hipSuccess ? MDN_OK : MDN_ERR_LAUNCH; }

// F(type tag, row length tag)
template <typename F> int dispatch(const mdn_shape *s, F &&f) {
    if (s->dtype == MDN_DTYPE_F32) {
        if (s->dk == 64) return f(float{}, std::integral_constant<int, 64>{});
        return f(float{}, std::integral_constant<int, 128>{});
    }
    if (s->dk == 64) return f(bf16_t{}, std::integral_constant<int, 64>{});
    return f(bf16_t{}, std::integral_constant<int, 128>{});
}

template <int N> bool kept_set(const mdn_kept *k, KeptSet<N> *s) {
    if (!k) return false;
    for (int i = 0; i < N; ++i) {
        if (!k[i].codes || !k[i].exponents) return false;
        s->t[i] = Kept{k[i].codes, k[i].exponents};
    }
    return true;
}

constexpr int kMaxCus = 1024; // of a device
size_t front_ws(const LayerDims &d) { return ((size_t)d.rows + (size_t)kMaxSlabs * d.H) * sizeof(float); }
size_t back_ws(int D) { return (size_t)kMaxCus * D * sizeof(float); }
bool misaligned(const void *p) { return reinterpret_cast<uintptr_t>(p) & 3u; }

} // namespace

} // namespace mdn

using namespace mdn;

extern "C" {

int mdn_kept_workspace_bytes(const mdn_shape *shape, size_t *bytes_out) {
    LayerDims ld;
    if (!bytes_out) return MDN_ERR_NULL;
    const int rc = check_layer(shape, &ld);
    if (rc) return rc;
    const size_t a = front_ws(ld), b = back_ws(shape->dk);
    *bytes_out = a > b ? a : b;
    return MDN_OK;
}

int mdn_keep(const mdn_shape *shape, const void *x, const mdn_kept *kept, void *stream) {
    LayerDims ld;
    KeptSet<1> ks;
    const int rc = check_layer(shape, &ld);
    if (rc) return rc;
    if (!x || !kept_set(kept, &ks)) return MDN_ERR_NULL;
    return dispatch(shape, [&](auto t, auto dim) {
        typedef decltype(t) T;
        constexpr int D = decltype(dim)::value;
        const Launch l = stream_launch(ld.rows, Rows<T, D>::RPW);
        hipLaunchKernelGGL((kept_copy_kernel<T, D, true>), dim3(l.grid), dim3(l.block), 0, static_cast<hipStream_t>(stream), ld,
                           static_cast<T *>(const_cast<void *>(x)), ks.t[0]);
        return status();
    });
}

int mdn_kept_values(const mdn_shape *shape, const mdn_kept *kept, void *x, void *stream) {
    LayerDims ld;
    KeptSet<1> ks;
    const int rc = check_layer(shape, &ld);
    if (rc) return rc;
    if (!x || !kept_set(kept, &ks)) return MDN_ERR_NULL;
    return dispatch(shape, [&](auto t, auto dim) {
        typedef decltype(t) T;
        constexpr int D = decltype(dim)::value;
        const Launch l = stream_launch(ld.rows, Rows<T, D>::RPW);
        hipLaunchKernelGGL((kept_copy_kernel<T, D, false>), dim3(l.grid), dim3(l.block), 0, static_cast<hipStream_t>(stream), ld, static_cast<T *>(x),
                           ks.t[0]);
        return status();
    });
}

int mdn_frontend_fwd_keep(const mdn_shape *shape, const void *x_q, const void *x_k, const void *x_v, const float *d, float eps, void *q, void *k,
                          void *v, const mdn_kept *kept, void *stream) {
    LayerDims ld;
    KeptSet<3> ks;
    const int rc = check_layer(shape, &ld);
    if (rc) return rc;
    if (!x_q || !x_k || !x_v || !d || !q || !k || !v || !kept_set(kept, &ks)) return MDN_ERR_NULL;
    return dispatch(shape, [&](auto t, auto dim) {
        typedef decltype(t) T;
        constexpr int D = decltype(dim)::value;
        const Launch l = stream_launch(ld.rows, Rows<T, D>::RPW);
        hipLaunchKernelGGL((frontend_fwd_kept_kernel<T, D, false>), dim3(l.grid), dim3(l.block), 0, static_cast<hipStream_t>(stream), ld,
                           static_cast<const T *>(x_q), static_cast<const T *>(x_k), static_cast<const T *>(x_v), ks, d, eps,
                           static_cast<T *>(q), static_cast<T *>(k), static_cast<T *>(v));
        return status();
    });
}

int mdn_frontend_fwd_kept(const mdn_shape *shape, const mdn_kept *kept, const float *d, float eps, void *q, void *k, void *v, void *stream) {
    LayerDims ld;
    KeptSet<3> ks;
    const int rc = check_layer(shape, &ld);
    if (rc) return rc;
    if (!d || !q || !k || !v || !kept_set(kept, &ks)) return MDN_ERR_NULL;
    return dispatch(shape, [&](auto t, auto dim) {
        typedef decltype(t) T;
        constexpr int D = decltype(dim)::value;
        const Launch l = stream_launch(ld.rows, Rows<T, D>::RPW);
        hipLaunchKernelGGL((frontend_fwd_kept_kernel<T, D, true>), dim3(l.grid), dim3(l.block), 0, static_cast<hipStream_t>(stream), ld,
                           static_cast<const T *>(nullptr), static_cast<const T *>(nullptr), static_cast<const T *>(nullptr), ks, d, eps,
                           static_cast<T *>(q), static_cast<T *>(k), static_cast<T *>(v));
        return status();
    });
}

int mdn_frontend_bwd_kept(const mdn_shape *shape, const mdn_kept *kept, const float *d, float eps, const void *dq, const void *dk, const void *dv,
                          void *dx_q, void *dx_k, void *dx_v, float *dd, void *workspace, size_t workspace_bytes, void *stream) {
    LayerDims ld;
    KeptSet<3> ks;
    int rc = check_layer(shape, &ld);
    if (rc) return rc;
    if (!d || !dq || !dk || !dv || !dx_q || !dx_k || !dx_v || !kept_set(kept, &ks) || (dd && !workspace)) return MDN_ERR_NULL;
    if (dd && misaligned(workspace)) return MDN_ERR_ALIGN;
    if (dd && workspace_bytes < front_ws(ld)) return MDN_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    float *rows = dd ? static_cast<float *>(workspace) : nullptr;
    rc = dispatch(shape, [&](auto t, auto dim) {
        typedef decltype(t) T;
        constexpr int D = decltype(dim)::value;
        const Launch l = stream_launch(ld.rows, Rows<T, D>::RPW);
        hipLaunchKernelGGL((frontend_bwd_kept_kernel<T, D>), dim3(l.grid), dim3(l.block), 0, s, ld, ks, d, eps, static_cast<const T *>(dq),
                           static_cast<const T *>(dk), static_cast<const T *>(dv), static_cast<T *>(dx_q), static_cast<T *>(dx_k),
                           static_cast<T *>(dx_v), rows);
        return status();
    });
    if (rc || !dd) return rc;
    const int tokens = (int)(ld.rows / (unsigned)ld.H), n = kept_slabs(ld.rows, ld.H);
    float *parts = n == 1 ? dd : rows + ld.rows;
    hipLaunchKernelGGL(sum_tokens_kernel, dim3(n), dim3(kSumThreads), 0, s, rows, parts, tokens, ld.H);
    if (n > 1) hipLaunchKernelGGL(sum_tokens_kernel, dim3(1), dim3(kSumThreads), 0, s, parts, dd, n, ld.H);
    return status();
}

int mdn_epilogue_fwd_keep(const mdn_shape *shape, const void *o, const void *g, const float *w, float eps, void *y, const mdn_kept *kept,
                          void *stream) {
    LayerDims ld;
    KeptSet<2> ks;
    const int rc = check_layer(shape, &ld);
    if (rc) return rc;
    if (!o || !g || !w || !y || !kept_set(kept, &ks)) return MDN_ERR_NULL;
    return dispatch(shape, [&](auto t, auto dim) {
        typedef decltype(t) T;
        constexpr int D = decltype(dim)::value;
        const Launch l = stream_launch(ld.rows, Rows<T, D>::RPW);
        hipLaunchKernelGGL((epilogue_fwd_keep_kernel<T, D>), dim3(l.grid), dim3(l.block), 0, static_cast<hipStream_t>(stream), ld,
                           static_cast<const T *>(o), static_cast<const T *>(g), ks, w, eps, static_cast<T *>(y));
        return status();
    });
}

int mdn_epilogue_bwd_kept(const mdn_shape *shape, const mdn_kept *kept, const float *w, float eps, const void *dy, void *d_o, void *dg, float *dw,
                          void *workspace, size_t workspace_bytes, void *stream) {
    LayerDims ld;
    KeptSet<2> ks;
    int rc = check_layer(shape, &ld);
    if (rc) return rc;
    if (!w || !dy || !d_o || !dg || !kept_set(kept, &ks) || (dw && !workspace)) return MDN_ERR_NULL;
    if (dw && misaligned(workspace)) return MDN_ERR_ALIGN;
    if (dw && workspace_bytes < back_ws(shape->dv)) return MDN_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    int parts = 0;
    rc = dispatch(shape, [&](auto t, auto dim) -> int {
        typedef decltype(t) T;
        constexpr int D = decltype(dim)::value;
        const Launch l = dw ? reduce_launch(ld.rows, Rows<T, D>::RPW) : stream_launch(ld.rows, Rows<T, D>::RPW);
        if (dw && l.grid > kMaxCus) return MDN_ERR_DEVICE;
        parts = l.grid;
        hipLaunchKernelGGL((epilogue_bwd_kept_kernel<T, D>), dim3(l.grid), dim3(l.block), 0, s, ld, ks, w, eps, static_cast<const T *>(dy),
                           static_cast<T *>(d_o), static_cast<T *>(dg), dw ? static_cast<float *>(workspace) : nullptr);
        return status();
    });
    if (rc || !dw) return rc;
    hipLaunchKernelGGL(sum_tokens_kernel, dim3(1), dim3(kSumThreads), 0, s, static_cast<const float *>(workspace), dw, parts, shape->dv);
    return status();
}

} // extern "C"
