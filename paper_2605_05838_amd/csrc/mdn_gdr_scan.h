// What the forward and the reverse scan of the gated delta rule have in common.
//
// A workgroup walks the chunks of one (sequence, value head) pair for 32 columns of the state, one barrier per chunk, with six waves:
//   waves 2, 3  the chain: 16 columns each, the state in their accumulators (see mdn_gdr.h);
//   waves 0, 1  what hangs on the chain without being part of it, for the same columns, and every store;
//   waves 4, 5  loads: the chunks ahead, HBM -> LDS without registers, into rings of kDepth chunks.
// (Waves are dealt to the four SIMDs in turn: the chain has SIMDs 2 and 3 to itself.)  The fragments of T and P go from memory straight
// into the registers of the one wave per 16 columns that wants them, asked for as soon as those of the chunk before are used up.
#pragma once
#include "mdn_gdr.h"

namespace mdn {

constexpr int kGdrThreads = 384, kGdrCols = 32;

// The tiles of a chunk that the loading waves (w2 = 0, 1) bring: [64][D] rows, permuted as GTile<T, LAYOUT> says
template <typename T, int D, bool PERMUTED> struct GLoad {
    static constexpr int E = 16 / (int)sizeof(T), CPR = D / E, COUNT = 64 * CPR / 128, BYTES = 64 * CPR * 16;
    unsigned off[COUNT];
    __device__ __forceinline__ void aim(unsigned row_elems, int w2, int lane, int last) {
#pragma unroll
        for (int u = 0; u < COUNT; ++u) {
            const int slot = (u * 2 + w2) * 64 + lane;
            if constexpr (PERMUTED) off[u] = GTile<T, D>::source(slot, row_elems * (unsigned)sizeof(T), last);
            else off[u] = (unsigned)min(slot / CPR, last) * row_elems * (unsigned)sizeof(T) + slot % CPR * 16;
        }
    }
    __device__ __forceinline__ void request(const T *src, const T *tile, int w2) const {
#pragma unroll
        for (int u = 0; u < COUNT; ++u) dma16(src, off[u], lds_addr(tile) + (u * 2 + w2) * 1024);
    }
};

// A wave's triangle fragments of one chunk
template <typename T> struct Triangle {
    typename Gd<T>::Frag f[Gd<T>::NF];
    __device__ __forceinline__ void load(const void *base, size_t blk, int lane) {
        const auto *p = static_cast<const typename Gd<T>::Frag *>(base) + blk * (Gd<T>::NF * 64) + lane;
#pragma unroll
        for (int i = 0; i < Gd<T>::NF; ++i) f[i] = p[i * 64];
    }
};
template <typename T, bool ON> struct TriangleIf : Triangle<T> {};
template <typename T> struct TriangleIf<T, false> {
    __device__ __forceinline__ void load(const void *, size_t, int) {}
};

// B fragments of N accumulator tiles, with their remainders (PRECISE)
template <typename T, int N, bool PRECISE> struct Frags {
    static constexpr int S = N / Gd<T>::KT;
    typename Gd<T>::Frag hi[S], lo[PRECISE ? S : 1];
    __device__ __forceinline__ void from(const f32x4 (&c)[N]) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            hi[s] = Gd<T>::frag(&c[s * Gd<T>::KT]);
            if constexpr (PRECISE) lo[s] = Gd<T>::rest(&c[s * Gd<T>::KT], hi[s]);
        }
    }
    // acc += a B, step s
    __device__ __forceinline__ f32x4 mma(typename Gd<T>::Frag a, int s, f32x4 acc) const {
        acc = gd_mma<T>(a, hi[s], acc);
        if constexpr (PRECISE) acc = gd_mma<T>(a, lo[s], acc);
        return acc;
    }
};

// [16 columns][N rows] of storage elements in LDS, in which a wave leaves its fragments: an element's row is its place
template <typename T, int N> struct Slate {
    static constexpr int LD = N + Gd<T>::E, SIZE = 16 * LD;
    static __device__ __forceinline__ void put(T *t, int s, int r, int kg, typename Gd<T>::Frag f) {
        *reinterpret_cast<typename Gd<T>::Frag *>(t + r * LD + s * Gd<T>::KS + kg * Gd<T>::E) = f;
    }
    static __device__ __forceinline__ typename Gd<T>::Frag get(const T *t, int s, int r, int kg) {
        return *reinterpret_cast<const typename Gd<T>::Frag *>(t + r * LD + s * Gd<T>::KS + kg * Gd<T>::E);
    }
};

// a slate of 64 tokens -> 16 columns of `rows` rows of a [tokens, H, dv] tensor
template <typename T> __device__ __forceinline__ void store_tokens(T *base, unsigned rs, const T *slate, int rows, int r, int kg) {
    constexpr int LD = Slate<T, 64>::LD;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto v = column4(slate, LD, 4 * kg, 16 * i, r);
        const int tok = 16 * i + r;
        if (tok < rows) __builtin_nontemporal_store(v, reinterpret_cast<decltype(column4(slate, LD, 0, 0, 0)) *>(at32(base, tok * rs + 4 * kg)));
    }
}

// A slate of DK rows of a state -> a chunk block of kept states: A fragments (row tile t, step of dv), [dv / KS][DK / 16] of them,
// cg: the 16-column group of the workgroup, col0: the workgroup's first column
template <typename T, int DK> __device__ __forceinline__ void store_state(T *block, const T *slate, int cg, int col0, int lane) {
    constexpr int LD = Slate<T, DK>::LD, NT = DK / 16;
    if constexpr (sizeof(T) == 2) { // two lane groups per tile: the other two are the other 16 columns'
        const int r = lane & 15, g = lane >> 4 & 1, up = lane >> 5;
#pragma unroll
        for (int tt = 0; tt < NT; tt += 2) {
            const int t = tt + up, dk = 32 * (t >> 1) + 4 * (t & 1) + 8 * (r & 3);
            const bf16_t *p = slate + (8 * g + (r >> 2)) * LD + dk;
            const bf16x8 v = tr_pair(p, p + 4 * LD);
            __builtin_nontemporal_store(v, reinterpret_cast<bf16x8 *>(block + (((size_t)(col0 >> 5) * NT + t) * 64 + (2 * cg + g) * 16 + r) * 8));
        }
    } else {
        const int r = lane & 15, kg = lane >> 4;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const f32x4 v = column4(slate, LD, 4 * kg, 16 * t, r);
            __builtin_nontemporal_store(v, reinterpret_cast<f32x4 *>(block + (((size_t)(col0 / 16 + cg) * NT + t) * 64 + lane) * 4));
        }
    }
}

// a wave's state tiles from and to a [dk][dv] fp32 tensor, column col + r
template <typename T, int NT> __device__ __forceinline__ void load_state(f32x4 (&S)[NT], const float *g, int dv, int col, int r, int kg) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) S[t][x] = g ? g[(size_t)(Gd<T>::row(t, 4 * kg) + x) * dv + col + r] : 0.f;
}
template <typename T, int NT> __device__ __forceinline__ void save_state(const f32x4 (&S)[NT], float *g, int dv, int col, int r, int kg) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) g[(size_t)(Gd<T>::row(t, 4 * kg) + x) * dv + col + r] = S[t][x];
}

} // namespace mdn
