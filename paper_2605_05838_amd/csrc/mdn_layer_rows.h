// What the kernels of the layer's elementwise operations share: rows of [B,T,H,d] tensors held 16 bytes (or less) a lane, the sums over a
// row, the walk over the rows, launch shapes and argument checks.
#pragma once
#include "../../include/mdn.h"
#include "mdn_device.h"
#include "mdn_kernels.h"

#include <hip/hip_runtime.h>

namespace mdn {

constexpr int LT = 256; // threads of the kernels without parameter gradients

// sigmoid: 1 / (1 + e^-x) by the reciprocal instruction (1 ulp) and one Newton step.  Compared for every fp32 value of e^-x
// from 0 to infinity, the quotient is bit for bit that of the IEEE division (ten instructions: the kernels were bound by
// them), denormal quotients to one unit in their last place.  The reciprocal flushes denormal results, which is why it is taken
// of 2^-32 times its argument; at e^-x = infinity its residual is not a number, which the maximum replaces.
// (The bare reciprocal, 16-bit storage: front end forward 33.6 us where it takes 35.7, adjoint 54.9 / 55.6; back end
// 18.7 / 18.7, 32.6 / 33.6.)
__device__ __forceinline__ float sigm(float x) {
    const float d = __builtin_fmaf(__expf(-x), 0x1p-32f, 0x1p-32f), r = __builtin_amdgcn_rcpf(d);
    const float e = fmaxf(__builtin_fmaf(-d, r, 1.f), -1.f);
    return __builtin_fmaf(r, e, r) * 0x1p-32f;
}

// This lane's E elements of a row of D: D / E lanes hold a row, 64 E / D rows a wave.  Tensors need no more than the alignment
// of their elements (a weight sliced out of a flat buffer): the vector types say so, and 16-byte accesses stay 16 bytes wide,
// which the hardware takes at any address.
template <typename T, int D, int E_> struct Row {
    static constexpr int E = E_, LPR = D / E, RPW = 64 / LPR;
    typedef bf16x8 __attribute__((aligned(2))) Half8;
    typedef f32x4 __attribute__((aligned(4))) Float4;
    float v[E];
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (sizeof(T) == 2 && E == 8) {
            const bf16x8 x = *reinterpret_cast<const Half8 *>(p);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = (float)x[e];
        } else if constexpr (sizeof(T) == 4 && E % 4 == 0) {
#pragma unroll
            for (int u = 0; u < E; u += 4) {
                const f32x4 x = *reinterpret_cast<const Float4 *>(p + u);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[u + e] = x[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = to_f32(p[e]);
        }
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (sizeof(T) == 2 && E == 8) {
            bf16x8 x;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = (bf16_t)v[e];
            *reinterpret_cast<Half8 *>(p) = x;
        } else if constexpr (sizeof(T) == 4 && E % 4 == 0) {
#pragma unroll
            for (int u = 0; u < E; u += 4) *reinterpret_cast<Float4 *>(p + u) = f32x4{v[u], v[u + 1], v[u + 2], v[u + 3]};
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] = from_f32<T>(v[e]);
        }
    }
    // sum of x over the lanes of a row, in every one of them
    static __device__ __forceinline__ float row_sum(float x) {
        static_assert(LPR == 8 || LPR == 16 || LPR == 32 || LPR == 64, "lanes of a row");
        if constexpr (LPR == 8) {
            x += dpp_move<0xB1>(x);         // quad_perm [1,0,3,2]
            x += dpp_move<0x4E>(x);         // quad_perm [2,3,0,1]
            return x + dpp_move<0x141>(x);  // row_half_mirror: the other quad of the 8 lanes
        }
        x = reduce16(x);
        if (LPR > 16) x = add_xor16(x);
        if (LPR > 32) x = add_xor32(x);
        return x;
    }
};

struct LayerDims {
    unsigned rows; // B*T*H
    int H;
};

// The rows of one lane: row0, row0 + step, ... and their heads (row % H, carried along).
struct RowWalk {
    unsigned row, step;
    int h, dh;
    __device__ __forceinline__ RowWalk(const LayerDims &d, int rows_per_wave, int lanes_per_row) {
        const unsigned waves = blockDim.x >> 6;
        row = (blockIdx.x * waves + wave_id()) * rows_per_wave + lane_id() / lanes_per_row;
        step = gridDim.x * waves * rows_per_wave;
        h = (int)(row % (unsigned)d.H);
        dh = (int)(step % (unsigned)d.H);
    }
    __device__ __forceinline__ void next(const LayerDims &d) {
        row += step;
        h += dh;
        h = h >= d.H ? h - d.H : h;
    }
};

inline int check_layer(const mdn_shape *s, LayerDims *d) {
    if (!s) return MDN_ERR_NULL;
    if (s->dtype != MDN_DTYPE_BF16 && s->dtype != MDN_DTYPE_F32) return MDN_ERR_DTYPE;
    if (s->B < 1 || s->T < 1 || s->H < 1 || s->H > 4096) return MDN_ERR_SHAPE;
    if (!((s->dk == 64 && s->dv == 64) || (s->dk == 128 && s->dv == 128))) return MDN_ERR_SHAPE;
    const long long rows = (long long)s->B * s->T * s->H;
    if (rows > 0x7fffffffLL) return MDN_ERR_SHAPE; // (more than 288 GB of tensors)
    d->rows = (unsigned)rows;
    d->H = s->H;
    return MDN_OK;
}

// launch shape of a row-streaming kernel: workgroups of 256 threads, at most 32 per CU
struct Launch { int grid, block; };
inline Launch stream_launch(unsigned rows, unsigned rows_per_wave) {
    const unsigned per = LT / 64 * rows_per_wave, need = (rows + per - 1) / per, most = 32u * (unsigned)num_cus();
    return Launch{(int)(need < most ? need : most), LT};
}
// the same for a kernel that ends in atomic adds on a few addresses: one workgroup per CU at most, of 1 024 threads once
// there are rows enough to give every CU one (below that, smaller workgroups reach more CUs)
inline Launch reduce_launch(unsigned rows, unsigned rows_per_wave) {
    const unsigned cus = (unsigned)num_cus();
    const unsigned waves = rows >= cus * 16u * rows_per_wave ? 16u : 4u, per = waves * rows_per_wave, need = (rows + per - 1) / per;
    return Launch{(int)(need < cus ? need : cus), (int)waves * 64};
}

} // namespace mdn
