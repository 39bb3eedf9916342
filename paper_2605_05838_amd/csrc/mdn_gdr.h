// What the kernels of the gated delta rule share.  Per (sequence, value head h, key head h / (H / Hk)), a_t = e^{g_t}:
//     e_t = v_t - a_t S_{t-1}^T k_t;   S_t = a_t S_{t-1} + beta_t k_t e_t^T;   o_t = scale S_t^T q_t
// and for a chunk of 64 tokens (G_i: inclusive sums of g inside the chunk, C its last token):
//     A_ij = e^{G_i - G_j} beta_j k_i.k_j  (j < i)     P_ij = e^{G_i - G_j} beta_j q_i.k_j  (j <= i)     T = (I + A)^-1
//     E = T (V - e^G K S0)       O = scale (e^G Q S0 + P E)       S_C = e^{G_C} S0 + (e^{G_C - G} beta K)^T E
// Adjoint (dO' = scale dO):
//     dE = P^T dO' + e^{G_C - G} beta K dS_C     dV = T^T dE     dS0 = e^{G_C} dS_C + (e^G Q)^T dO' - (e^G K)^T dV
//
// Every column of a state evolves by itself, and a wave of the scans owns 16 of them.  Its state tiles are MFMA accumulators (a lane
// has 4 rows of one column), and which rows those are is the kernel's choice: with rows 8 kg .. 8 kg + 7 of every 32 in lane
// group kg (`Gd::row`), a lane's accumulators of two tiles, rounded, ARE the B fragment of the product that contracts over those rows.
// So states, corrections and their adjoints go from product to product without leaving the registers: no LDS round trip and
// no barrier is on the chain of a chunk, whose products take their A operands from token tiles in LDS.
//
// What is rounded to the storage type: what the tensors hold, the kept states and adjoints, and the products' operands (S, T, P, V - e^G K S, E, D, dE,
// dV, W); sums, decays, the inverse and the states along a chain are fp32.  With 16 bits against fp64, rms: o, e, dq, dk 2.9e-3, dv 1.7e-3, dg 2.4e-3 to
// 4.2e-3, dbeta 2.3e-3 to 3.6e-3 (64 to 1 000 tokens, adjoints of the final states of any size), where rounding an exact result once leaves 1.7e-3; fp32
// products run at an eighth of the rate or less, and operands of value + remainder, which states that leave the call in 32 bits are carried with (3e-6),
// take two or three products for one.
#pragma once
#include "mdn_device.h"
#include "mdn_kernels.h"
#include "mdn_scan_tiles.h"

namespace mdn {

struct GdrDims {
    int B, T, H, Hk;   // B sequences of T tokens; packed batches: B sequences of their own lengths, T tokens together
    int N, nchunks;    // chunks of the longest sequence, of all sequences
    int c0, cn;        // sequences of equal lengths: a launch's chunks of each, [c0, c0 + cn) of the N
    int dk, dv, dtype; // MDN_DTYPE_*
    float scale;
    const SeqEntry *seqs;     // packed batches: [B], longest first; otherwise null
    const ChunkEntry *chunks; // packed batches: [nchunks]; otherwise null
};

// Chunk-local operands of the scans, one block per (sequence, head, chunk): coef = {e^G | e^{G_C - G} beta | unused}, 64 floats
// each, 256 together; masked matrices as A fragments in the order in which a wave loads them (Gd::low, Gd::up; a fragment is 1 KB).
// _lo: what the rounding to 16 bits dropped, rounded again.  Any may be null: not written.
constexpr int kGdrCoef = 256;
struct GdrLocalArgs {
    const void *q, *k;
    const float *g, *beta;
    float *coef;
    void *T, *T_lo, *P;            // forward
    void *TT, *TT_lo, *PT, *PT_lo; // reverse scan
};
struct GdrScanFwdArgs {
    const void *q, *k, *v; // v: e where states are reconstructed
    const float *coef;
    const void *T, *T_lo, *P;
    const float *S0;
    void *o, *e, *states; // e, states may be null
    float *S_final;       // may be null
    int touch;            // whether later chunks are brought into the L2; the launch sets it
};
struct GdrScanBwdArgs {
    const void *q, *k, *dO;
    const float *coef;
    const void *TT, *TT_lo, *PT, *PT_lo;
    const float *dS_final; // may be null
    void *dv, *dstates;    // dstates: adjoints of the chunk-END states
    float *dS0;            // may be null
};
struct GdrGradArgs {
    const void *q, *k, *e, *dO, *dv;
    const float *g, *beta;
    const void *states, *dstates;
    void *sums; // H > Hk: gdr_sums_bytes() of workspace; otherwise null
    void *dq, *dk, *dg, *dbeta;
    bool f32_gates; // dg, dbeta in fp32, not in the storage type
};
struct GdrStepArgs {
    const void *q, *k, *v;
    const float *g, *beta;
    float *S;
    void *o;
};

hipError_t launch_gdr_local(const GdrDims &d, const GdrLocalArgs &a, hipStream_t s);
// precise: the products that lead to a state take their 16-bit operands as value + remainder
hipError_t launch_gdr_scan_fwd(const GdrDims &d, const GdrScanFwdArgs &a, bool precise, hipStream_t s);
hipError_t launch_gdr_rebuild(const GdrDims &d, const GdrScanFwdArgs &a, hipStream_t s);
hipError_t launch_gdr_scan_bwd(const GdrDims &d, const GdrScanBwdArgs &a, bool precise, hipStream_t s);
hipError_t launch_gdr_grad(const GdrDims &d, const GdrGradArgs &a, hipStream_t s);
hipError_t launch_gdr_step(const GdrDims &d, const GdrStepArgs &a, hipStream_t s);

// bytes of one fragment set (a triangle of a 64 x 64 matrix)
inline size_t gdr_triangle_bytes(int dtype) { return dtype == 1 ? 10240 : 6144; }

// 32-bit sums of dq, dk and two triangles over the value heads of a key head, per chunk and key head
inline size_t gdr_sums_bytes(int dk) { return (size_t)(2 * 64 * dk + 2 * 12 * 256) * sizeof(float); }

// ---- layouts
template <typename T> struct Gd;
template <> struct Gd<bf16_t> {
    typedef bf16x8 Frag;
    static constexpr int E = 8, KS = 32, KT = 2; // elements of a fragment's lane; contraction of a step; accumulator tiles of a step
    static constexpr int NF = 6;                 // fragments of a triangle
    // the row (of 64 tokens, of dk) that row m of tile t stands for
    static __device__ __forceinline__ int row(int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); }
    // fragment (row tile t, step s) of a lower triangle: steps 0 .. last(t); of an upper one: steps first(t) ..
    static constexpr __host__ __device__ int last(int t) { return t >> 1; }
    static constexpr __host__ __device__ int first(int t) { return t >> 1; }
    static constexpr __host__ __device__ int low(int t, int s) { return t < 2 ? t : 2 * (t - 1) + s; }
    static constexpr __host__ __device__ int up(int t, int s) { return t < 2 ? 2 * t + s : t + 2; }
    static __device__ __forceinline__ Frag frag(const f32x4 *c) { // of one step's tiles
        return Frag{(bf16_t)c[0][0], (bf16_t)c[0][1], (bf16_t)c[0][2], (bf16_t)c[0][3],
                    (bf16_t)c[1][0], (bf16_t)c[1][1], (bf16_t)c[1][2], (bf16_t)c[1][3]};
    }
    // what frag() dropped
    static __device__ __forceinline__ Frag rest(const f32x4 *c, Frag f) {
#pragma clang fp contract(off) // (of the value as it was rounded to 32 bits, wherever the compiler inlines this: results do not depend on it)
        Frag r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = (bf16_t)(c[e >> 2][e & 3] - (float)f[e]);
        return r;
    }
};
template <> struct Gd<float> {
    typedef f32x4 Frag;
    static constexpr int E = 4, KS = 16, KT = 1;
    static constexpr int NF = 10;
    static __device__ __forceinline__ int row(int t, int m) { return 16 * t + m; }
    static constexpr __host__ __device__ int last(int t) { return t; }
    static constexpr __host__ __device__ int first(int t) { return t; }
    static constexpr __host__ __device__ int low(int t, int s) { return t * (t + 1) / 2 + s; }
    static constexpr __host__ __device__ int up(int t, int s) { return 4 * t - t * (t - 1) / 2 + s - t; }
    static __device__ __forceinline__ Frag frag(const f32x4 *c) { return c[0]; }
    static __device__ __forceinline__ Frag rest(const f32x4 *, Frag) { return Frag{0.f, 0.f, 0.f, 0.f}; }
};

// A [64][D] token tile in LDS.  The 16-byte pieces of a row are permuted by XOR with a number that differs between the 16
// rows of a fragment read and spreads the rows of a transposing read: both are free of bank conflicts.
template <typename T, int D> struct GTile {
    static constexpr int E = Gd<T>::E, CPR = D / E, PIECES = 64 * CPR, BYTES = PIECES * 16;
    static __device__ __forceinline__ int turn(int row) {
        if constexpr (sizeof(T) == 4) return row & 15 & (CPR - 1);
        else if constexpr (CPR >= 16) return (row & 3) << 2 | (row >> 3 & 3);
        else if constexpr (CPR == 8) return (row >> 1 & 1) << 2 | (row >> 3 & 3);
        else return 0;
    }
    // the lane's 16 bytes of slot `slot` (slot = 64 u + lane of instruction u), as a byte offset from the tile's first row; rs: bytes
    // between rows, last: the last row that exists (rows behind it receive copies of it)
    static __device__ __forceinline__ unsigned source(int slot, unsigned rs, int last) {
        const int row = slot / CPR, pc = (slot % CPR) ^ turn(row);
        return (unsigned)min(row, last) * rs + pc * 16;
    }
    template <typename P> static __device__ __forceinline__ P *at(P *tile, int row, int col) { // col: multiple of what is moved at once
        return tile + row * D + ((col / E) ^ turn(row)) * E + col % E;
    }
    // row `row`, elements KS s + E kg ..: the tile as [row][contraction] operand
    static __device__ __forceinline__ typename Gd<T>::Frag row_frag(const T *tile, int row, int s, int kg) {
        return *reinterpret_cast<const typename Gd<T>::Frag *>(at(tile, row, (s * 4 + kg) * E));
    }
    // column Gd::row(t, r), rows KS s + E kg ..: the transposed tile as [column][contraction] operand
    static __device__ __forceinline__ typename Gd<T>::Frag col_frag(const T *tile, int t, int s, int r, int kg) {
        if constexpr (sizeof(T) == 2) {
            const int row = 32 * s + 8 * kg + (r >> 2), col = 32 * (t >> 1) + 8 * (r & 3) + 4 * (t & 1);
            return tr_pair(at(tile, row, col), at(tile, row + 4, col));
        } else {
            f32x4 v;
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = *at(tile, 16 * s + 4 * kg + x, 16 * t + r);
            return v;
        }
    }
    // the same for column 16 t + r
    static __device__ __forceinline__ typename Gd<T>::Frag column_frag(const T *tile, int t, int s, int r, int kg) {
        if constexpr (sizeof(T) == 2) {
            const int row = 32 * s + 8 * kg + (r >> 2), col = 16 * t + 4 * (r & 3);
            return tr_pair(at(tile, row, col), at(tile, row + 4, col));
        } else {
            return col_frag(tile, t, s, r, kg);
        }
    }
};

// 4 rows row0 .. row0 + 3 of column col0 + r of a matrix in LDS kept [row][column] with row length ld
__device__ __forceinline__ f32x4 column4(const float *m, int ld, int row0, int col0, int r) {
    f32x4 v;
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = m[(row0 + x) * ld + col0 + r];
    return v;
}
__device__ __forceinline__ bf16x4 column4(const bf16_t *m, int ld, int row0, int col0, int r) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    const bf16_t *p = m + (row0 + (r >> 2)) * ld + col0 + (r & 3) * 4;
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p)));
}
// the lane's E rows E kg of step s of column col0 + r: a B fragment that contracts over rows
__device__ __forceinline__ bf16x8 column_frag(const bf16_t *m, int ld, int s, int kg, int col0, int r) {
    return __builtin_shufflevector(column4(m, ld, 32 * s + 8 * kg, col0, r), column4(m, ld, 32 * s + 8 * kg + 4, col0, r), 0, 1, 2, 3, 4, 5,
                                   6, 7);
}
__device__ __forceinline__ f32x4 column_frag(const float *m, int ld, int s, int kg, int col0, int r) {
    return column4(m, ld, 16 * s + 4 * kg, col0, r);
}

template <typename T> __device__ __forceinline__ f32x4 gd_mma(typename Gd<T>::Frag a, typename Gd<T>::Frag b, f32x4 c) {
    return Op<T>::mma(a, b, c);
}

// A lane's reads of such a tile, as few byte offsets that are formed once: what the permutation adds depends on the lane and on the step (rows
// as rows) or on the 32-column part (rows as contraction) alone, everything else is a constant of the instruction.
template <typename T, int D> struct TileReader {
    typedef Gd<T> G;
    typedef typename G::Frag Frag;
    static constexpr int NR = D / G::KS, NC = sizeof(T) == 2 ? D / 32 : 1;
    unsigned ro[NR], co[NC];
    int r, kg;
    __device__ __forceinline__ TileReader(int r_, int kg_) : r(r_), kg(kg_) {
        const T *z = nullptr;
#pragma unroll
        for (int s = 0; s < NR; ++s) ro[s] = (unsigned)(size_t)GTile<T, D>::at(z, G::row(0, r), (s * 4 + kg) * G::E);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int p = 0; p < NC; ++p) co[p] = (unsigned)(size_t)GTile<T, D>::at(z, 8 * kg + (r >> 2), 32 * p + 8 * (r & 3));
        }
    }
    // GTile::row_frag of row Gd::row(t, r)
    __device__ __forceinline__ Frag row_frag(const T *tile, int t, int s) const {
        return *reinterpret_cast<const Frag *>(reinterpret_cast<const char *>(tile) + ro[s] + G::row(t, 0) * D * (int)sizeof(T));
    }
    // GTile::col_frag
    __device__ __forceinline__ Frag col_frag(const T *tile, int t, int s) const {
        if constexpr (sizeof(T) == 2) {
            const bf16_t *p = reinterpret_cast<const bf16_t *>(reinterpret_cast<const char *>(tile) + co[t >> 1] + (32 * s * D + 4 * (t & 1)) * 2);
            return tr_pair(p, p + 4 * D);
        } else {
            return GTile<T, D>::col_frag(tile, t, s, r, kg);
        }
    }
};

// one (sequence, value head) pair of a scan
struct GdrSeq {
    size_t v, k;  // its first token as a row of the [tokens, H] and [tokens, Hk] tensors
    size_t blk;   // its first chunk block
    size_t state; // its index in the [sequences, H] state tensors
    int len, n;   // tokens, chunks
};
__device__ __forceinline__ GdrSeq gdr_seq(const GdrDims &d, int bh) {
    const int b = bh / d.H, h = bh % d.H, hk = h / (d.H / d.Hk);
    GdrSeq q;
    if (d.seqs) {
        SeqEntry e = d.seqs[b];
        e.t0 = __builtin_amdgcn_readfirstlane(e.t0);
        e.len = __builtin_amdgcn_readfirstlane(e.len);
        e.cb = __builtin_amdgcn_readfirstlane(e.cb);
        e.idx = __builtin_amdgcn_readfirstlane(e.idx);
        q.n = (e.len + 63) >> 6;
        q.len = e.len;
        q.v = (size_t)e.t0 * d.H + h;
        q.k = (size_t)e.t0 * d.Hk + hk;
        q.blk = (size_t)e.cb * d.H + (size_t)h * q.n;
        q.state = (size_t)e.idx * d.H + h;
    } else {
        const size_t t0 = (size_t)b * d.T + (size_t)d.c0 * 64;
        q.n = d.cn;
        q.len = min(d.T - d.c0 * 64, d.cn * 64);
        q.v = t0 * d.H + h;
        q.k = t0 * d.Hk + hk;
        q.blk = (size_t)bh * d.N + d.c0;
        q.state = bh;
    }
    return q;
}
// chunk `c` of a chunk-parallel launch (of all sequences), head h: first token, chunk block, tokens
struct GdrChunk {
    size_t tok, blk;
    int rows;
};
__device__ __forceinline__ GdrChunk gdr_chunk(const GdrDims &d, int c, int h) {
    GdrChunk p;
    if (d.chunks) {
        const ChunkEntry e = d.chunks[c];
        p.tok = (size_t)e.t0;
        p.blk = (size_t)e.blk + (size_t)h * e.N;
        p.rows = e.rows;
    } else {
        const int b = c / d.cn, n = d.c0 + c % d.cn;
        p.tok = (size_t)b * d.T + (size_t)n * 64;
        p.blk = ((size_t)b * d.H + h) * d.N + n;
        p.rows = min(64, d.T - n * 64);
    }
    return p;
}

// Decays of a chunk.  lane = token: log2 of the decay up to and including it as a sum of two floats, hi a multiple of 1/16 (its sums are
// exact) and lo small, so that the decay between two tokens keeps its relative accuracy behind however strong a decay before them:
// e^{G_i - G_j} = 2^(hi_i - hi_j) 2^(lo_i - lo_j).  Decays below 2^-200 a token count as 2^-200 (both are zero in fp32); tokens behind the
// last one have decay 1.
struct GdrDecay {
    float hi, lo;
    static __device__ __forceinline__ float pow2(float hi, float lo) { return __builtin_amdgcn_exp2f(hi) * __builtin_amdgcn_exp2f(lo); }
    __device__ __forceinline__ void sums(float g, int lane) {
        float x = g * 1.44269504f;
        x = x < -200.f ? -200.f : x; // (NaN stays)
        hi = __builtin_rintf(x * 16.f) * 0.0625f;
        lo = x - hi;
#pragma unroll
        for (int n = 1; n < 64; n *= 2) {
            const float h = __shfl_up(hi, n), l = __shfl_up(lo, n);
            hi += lane >= n ? h : 0.f;
            lo += lane >= n ? l : 0.f;
        }
    }
};

} // namespace mdn
