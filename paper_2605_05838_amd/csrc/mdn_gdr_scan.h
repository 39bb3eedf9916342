// What the forward and the reverse scan of the gated delta rule have in common.
//
// A workgroup walks the chunks of one (sequence, value head) pair for NCG groups of 16 columns of the state, one step per chunk, with
// four kinds of waves:
//   2 waves       beside the chain: what hangs on it without being part of it;
//   NCG waves     the chain: the state in their accumulators (see mdn_gdr.h); in fp32 and with remainders two waves to 16 columns (CW);
//   2 waves       loads: the chunks ahead, HBM -> LDS without registers, into rings;
//   2 waves       stores, out of LDS, and lines for later (GdrTouch); without rings (gdr_ring) the loading waves, whose loads are then not
//                 beside the products.
// A chain wave is bound by its LDS instructions, ~26 clocks each, most of them reads of A operands: 2 050 clocks a step at d = 128 in 16
// bits, 3 650 with remainders.  Two waves to 16 columns each form the products of half of the tokens with the whole state, whose other half
// they find in LDS since the step's barrier, hand them to the other one, and then have all they need for half of the next state; the small
// products with T in between both form.
// The chain loads nothing: the fragments of T, asked for by the wave that wants them as soon as those of the chunk before were used up,
// came back 2 000 clocks later, behind all of the step's tiles.  A chunk's tiles come 1 300 clocks and more after the request, so that two
// chunks are on their way while one is worked on: rings of three (of two: 2 350 clocks a step where three take 1 340).
#pragma once
#include "mdn_gdr.h"
#include "mdn_scan_rules.h"

namespace mdn {

// Whether LDS holds rings of chunks: not for 32-bit rows of 128, or of 64 with 32 columns.
template <typename T, int DK, int NCG> constexpr bool gdr_ring() { return sizeof(T) == 2 || (DK == 64 && NCG == 1); }

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

// A triangle's fragments of one chunk (or 1 KB of coefficients): memory -> LDS as they lie there
template <int BYTES> __device__ __forceinline__ void load_block(const void *base, size_t blk, void *to, int w2, int lane) {
    const char *p = static_cast<const char *>(base) + blk * BYTES;
    for (int u = w2; u < BYTES / 1024; u += 2) dma16(p, u * 1024 + lane * 16, lds_addr(to) + u * 1024);
}

// The operands of chunks further on than the loads, brought into the L2 by the storing waves: four bytes of every 64, each workgroup of a
// (sequence, head) pair its share of the lanes.  A CU has only so many lines on their way at a time, and all of a pair's workgroups ask for
// the same ones at the same time, so that every load took as long as one from HBM.
template <int N> struct GdrTouch { // N: places per lane (none: nothing is brought)
    const char *at[N ? N : 1];
    ptrdiff_t step[N ? N : 1];
    int end[N ? N : 1], p[N ? N : 1]; // a lane's lines are in the chunks before `end`
    // part: this wave's number among the `parts` storing waves of the pair
    __device__ __forceinline__ void aim(int part, int parts, int lane) {
#pragma unroll
        for (int u = 0; u < N; ++u) p[u] = (u * parts + part) * 64 + lane, end[u] = 0, at[u] = nullptr, step[u] = 0;
    }
    // a tensor's share: `rows` rows of `bytes`, `stride` apart, per chunk, the next chunk's `chunk` bytes on; `last`: the last row of the
    // last chunk
    __device__ __forceinline__ void add(const void *t, int rows, int bytes, ptrdiff_t stride, ptrdiff_t chunk, int chunks, int last) {
        const int per_row = bytes / 64;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int row = p[u] / per_row;
            if (p[u] >= 0 && row < rows) {
                at[u] = static_cast<const char *>(t) + row * stride + p[u] % per_row * 64;
                step[u] = chunk;
                end[u] = row > last ? chunks - 1 : chunks;
            }
            p[u] -= rows * per_row;
        }
    }
    // (as LDS transfers, which nothing has to wait for: dst is 256 bytes that nobody reads)
    __device__ __forceinline__ void chunk(int n, const void *dst) const {
#pragma unroll
        for (int u = 0; u < N; ++u)
            if (n >= 0 && n < end[u])
                asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dword %0, off"
                             :
                             : "v"(at[u] + n * step[u]), "s"(__builtin_amdgcn_readfirstlane((int)lds_addr(dst)))
                             : "memory", "m0");
    }
};
// places per lane for `lines` lines of 64 bytes and a row of dv elements in each of 64 rows, whether dv is 64 or 128
constexpr int touch_places(int lines, int bytes, int cols) {
    const int a = (lines + 64 * bytes - 1) / (64 / cols * 128) + 1, b = (lines + 128 * bytes - 1) / (128 / cols * 128) + 1;
    return a > b ? a : b;
}

// Everything asked for so far is there, and the compiler knows: it otherwise waits inside a loop for what was requested in front of it.
__device__ __forceinline__ void all_arrived() { __builtin_amdgcn_s_waitcnt(0x0f70); } // vmcnt(0)

// the slot of a ring of N that step n + 1 uses after step n's
template <int N> __device__ __forceinline__ int next_slot(int s) { return s + 1 == N ? 0 : s + 1; }

// fragment i of a triangle in LDS
template <typename T> __device__ __forceinline__ typename Gd<T>::Frag tri_frag(const T *tri, int i, int lane) {
    return *reinterpret_cast<const typename Gd<T>::Frag *>(tri + (i * 64 + lane) * Gd<T>::E);
}

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

// Stores go through buffer descriptors: what lies behind the last row is dropped by the bounds check.
typedef unsigned gdr_u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ __amdgpu_buffer_rsrc_t out_rows(void *base, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(base, 0, (int)bytes, 0x00020000);
}
template <int AUX, typename V> __device__ __forceinline__ void put16(__amdgpu_buffer_rsrc_t to, unsigned at, V v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(gdr_u32x4, v), to, at, 0, AUX);
}

// NG slates of LD rows, one after the other -> 32 tokens from token t0 on of a chunk of a [tokens, H, dv] tensor (`to`: from its first
// row and the first of the 16 NG columns on; rs: bytes between rows), whole rows of these columns at a time (32 bytes of a row and, later,
// the other 32 cost HBM two writes).  AUX: 2 for non-temporal
template <typename T, int NG, int LD, int AUX = 2>
__device__ __forceinline__ void store_tokens(__amdgpu_buffer_rsrc_t to, unsigned rs, const T *slates, int slate_t0, int t0, int r, int kg) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int pc = NG == 2 ? kg : kg & 1, tok = 16 * (NG == 2 ? i : kg >> 1) + r; // 16-byte piece of the row, token
            const T *p = slates + (8 * pc + (r >> 2)) * LD + slate_t0 + tok - r + 4 * (r & 3);
            put16<AUX>(to, (unsigned)(t0 + tok) * rs + 16 * pc, tr_pair(p, p + 4 * LD));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int pc = kg; pc < 4 * NG; pc += 4)
                put16<AUX>(to, (unsigned)(t0 + 16 * i + r) * rs + 16 * pc, column4(slates, LD, 4 * pc, slate_t0 + 16 * i, r));
    }
}

// NG slates of DK rows of a state, 16 columns each from column `col` on -> a chunk block of kept states: A fragments (row tile t, step of
// dv), [dv / KS][DK / 16] of them.  By two waves (w = 0, 1).
template <typename T, int DK, int NG>
__device__ __forceinline__ void store_state(__amdgpu_buffer_rsrc_t block, const T (&slates)[NG][Slate<T, DK>::SIZE], int w, int col, int lane) {
    constexpr int LD = Slate<T, DK>::LD, NT = DK / 16;
    const int r = lane & 15, kg = lane >> 4;
    if constexpr (sizeof(T) == 2 && NG == 2) { // whole fragments, every other one
        const T *p = slates[0] + (8 * kg + (r >> 2)) * LD + 8 * (r & 3); // (the second slate's columns are rows 16 ..: one after the other)
#pragma unroll
        for (int tt = 0; tt < NT; tt += 2) {
            const int t = tt + w;
            const T *x = p + 32 * (t >> 1) + 4 * (t & 1);
            put16<2>(block, (unsigned)((((col >> 5) * NT + t) * 64 + lane) * 16), tr_pair(x, x + 4 * LD));
        }
    } else if constexpr (sizeof(T) == 2) { // half of every fragment: two lane groups per tile
        const int g = kg & 1, half = col >> 3 & 2;
        const T *p = slates[0] + (8 * g + (r >> 2)) * LD + 8 * (r & 3);
#pragma unroll
        for (int tt = 0; tt < NT; tt += 4) {
            const int t = tt + 2 * w + (kg >> 1);
            const T *x = p + 32 * (t >> 1) + 4 * (t & 1);
            put16<2>(block, (unsigned)((((col >> 5) * NT + t) * 64 + (half + g) * 16 + r) * 16), tr_pair(x, x + 4 * LD));
        }
    } else {
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int tt = 0; tt < NT; tt += 2) {
                const int t = tt + w;
                put16<2>(block, (unsigned)((((col / 16 + g) * NT + t) * 64 + lane) * 16), column4(slates[g], LD, 4 * kg, 16 * t, r));
            }
    }
}

// Two waves of the same 16 columns wait for each other: `mine` says that this one's fragments of step n are in LDS (a wave's LDS
// operations are done in order), and it goes on when the other one's are.  Both are waves of one workgroup: the wait ends.
__device__ __forceinline__ void say(int *mine, int n) {
    asm volatile("" : : : "memory");
    *const_cast<volatile int *>(mine) = n + 1;
    asm volatile("" : : : "memory");
}
__device__ __forceinline__ void wait_for(const int *other, int n) {
    while (__builtin_amdgcn_readfirstlane(*const_cast<const volatile int *>(other)) <= n) {}
    asm volatile("" : : : "memory");
}

// a wave's state tiles (from tile T0 on) from and to a [dk][dv] fp32 tensor, column col + r
template <typename T, int T0 = 0, int NT> __device__ __forceinline__ void load_state(f32x4 (&S)[NT], const float *g, int dv, int col, int r, int kg) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) S[t][x] = g ? g[(size_t)(Gd<T>::row(T0 + t, 4 * kg) + x) * dv + col + r] : 0.f;
}
template <typename T, int T0 = 0, int NT> __device__ __forceinline__ void save_state(const f32x4 (&S)[NT], float *g, int dv, int col, int r, int kg) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) g[(size_t)(Gd<T>::row(T0 + t, 4 * kg) + x) * dv + col + r] = S[t][x];
}

// see gdr_bytes
inline size_t gdr_call_bytes(const GdrDims &d, int key_rows, int value_rows, bool states) {
    return gdr_bytes((size_t)d.nchunks * d.H, d.dk, d.dv, key_rows, value_rows, states);
}

// which of its two forms a scan takes: see sixteen_columns
inline bool gdr_one_group(const GdrDims &d) {
    return sixteen_columns(d.B, d.seqs ? d.nchunks : 0, d.N, d.H, d.dv, num_cus());
}

} // namespace mdn
