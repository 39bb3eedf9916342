// Gated delta rule, gradients of q, k, g and beta, chunk by chunk (dV is the reverse scan's).  S the state at the chunk's start, D the adjoint
// of the one at its end, dO' = scale dO, c_ij = e^{G_i - G_j} (i >= j), ec_j = e^{G_C - G_j}; per value head
//     W1 = c (dO' E^T) diag(beta)  (j <= i)      W2 = -c (dV E^T) diag(beta)  (j < i)
//     Z_ij = (W1_ij q_i.k_j + W2_ij k_i.k_j) / beta_j        b_j = ec_j k_j.(D E_j)        a_i = e^{G_i} (q_i.(S dO'_i) - k_i.(S dV_i))
//     dbeta_j = sum_{i >= j} Z_ij + b_j
//     dg_t = sum_{i >= t > j} beta_j Z_ij + sum_{i >= t} a_i + sum_{j < t} beta_j b_j + e^{G_C} <D, S>
// and with sums over the value heads of the key head
//     dq = sum e^G dO' S^T + (sum W1) K        dk = sum (beta ec E D^T - e^G dV S^T) + (sum W2) K + (sum W1)^T Q + (sum W2)^T K
// W1 and W2 are summed in 32 bits before their one rounding: what cancels between heads leaves no rounding behind, and the heads share
// these products.  The pairs of dg_t are sums of Z, taken from fp32 products: formed out of q.dq and k.dk instead, pairs that cancel in exact
// arithmetic would leave the roundings of W behind.  They are those with i >= t > j and no others, tile by tile (row sums, column sums, and in a
// tile on the diagonal sums over the rows from t on): all of them carry the decay of token t, so that dg_t is as exact behind a strong decay, and 0
// where the decay is; as a running difference of all column sums and all row sums it would be off by the rounding of what the others leave.
// One workgroup of four waves per (chunk, key head), which goes through its value heads; the states' parts of dq, dk and W1, W2 are summed in
// workspace that only their own thread touches (in registers they would spill others).
// A wave owns 32 of dk (with half of the tokens at dk = 64): its rows of S, D, K^T and Q^T are its A operands, straight
// from memory or out of the K, Q tiles by transposing reads, tokens are the B operands.  E, dO and dV come by 64 columns of dv at a time,
// so that two workgroups share a CU and one loads while the other multiplies.
// Bound by HBM: 176 KB a chunk and head at d = 128 (64 of them the two states), 3.9 TB/s of the copy's 5.1.
#include "mdn_coef.h"
#include "mdn_gdr.h"

namespace mdn {

namespace {

// the (row tile a, column tile b) pairs of wave w: as in the chunk-local kernel
constexpr unsigned kPairs[4] = {0x0dcu, 0x5feu, 0x98u, 0x4au};

__device__ __forceinline__ float dot(bf16x8 x, bf16x8 y) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (float)x[e] * (float)y[e];
    return s;
}
__device__ __forceinline__ float dot(f32x4 x, f32x4 y) { return x[0] * y[0] + x[1] * y[1] + x[2] * y[2] + x[3] * y[3]; }

template <typename T, int DK, int DV, bool SHARED> __global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void gdr_grad_kernel(GdrDims d, GdrGradArgs a, int first) {
    typedef Gd<T> G;
    typedef typename G::Frag Frag;
    typedef GTile<T, DK> TileK;
    typedef GTile<T, 64> TileV;
    constexpr int E = G::E, S64 = 64 / G::KS, SK = DK / G::KS, NP = DK / 32; // NP: 32-row parts of dk
    constexpr int NI = NP, I0 = 4 / NI; // token tiles of a wave (DK = 128: all four); waves that share a part
    constexpr int EARLY = sizeof(T) == 4 ? 0 : SHARED && DK + DV == 256 ? 1 : 2; // steps whose state fragments are asked for early (registers)
    static_assert(NI * I0 == 4 && (DK == 64 || DK == 128) && (DV == 64 || DV == 128), "sizes");
    __shared__ __align__(16) T s_k[64 * DK], s_q[64 * DK];
    __shared__ __align__(16) T s_e[64 * 64], s_do[64 * 64], s_dv[64 * 64]; // halves of E, dO, dV
    __shared__ __align__(16) T s_w1[64 * 64], s_w2[64 * 64];               // W1, W2 kept [j][i]
    __shared__ __align__(16) float s_hi[64], s_lo[64], s_be[64], s_eg[64], s_ec[64];
    __shared__ float s_row[4][64], s_col[4][64], s_a[4][64], s_b[4][64], s_tr[4];

    const int id = first + (int)blockIdx.x, hk = id % d.Hk, shared = SHARED ? d.H / d.Hk : 1;
    GdrChunk p = gdr_chunk(d, id / d.Hk, hk * shared);
    const int rows = p.rows;
    const unsigned rsk = (unsigned)(d.Hk * DK), rsv = (unsigned)(d.H * DV);
    const size_t key = (p.tok * d.Hk + hk) * DK;
    auto tile = [&](auto layout, T *to, const T *src, unsigned rs) { // by all four waves
        typedef decltype(layout) L;
        const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(wave_id());
#pragma unroll
        for (int u = 0; u < L::CPR / 4; ++u) {
            const int slot = (u * 4 + w) * 64;
            dma16(src, L::source(slot + lane, rs * (unsigned)sizeof(T), rows - 1), lds_addr(to) + slot * 16);
        }
    };
    tile(TileK{}, s_k, static_cast<const T *>(a.k) + key, rsk);
    tile(TileK{}, s_q, static_cast<const T *>(a.q) + key, rsk);

    for (int hs = 0; hs < shared; ++hs) {
        // (from values that the compiler cannot see through: it would otherwise keep every address of the loop in registers)
        int lane = lane_id(), w = wave_id();
        asm volatile("" : "+v"(lane), "+v"(w));
        w = __builtin_amdgcn_readfirstlane(w);
        const int r = lane & 15, kg = lane >> 4;
        const int part = w % NP, it0 = w / NP * NI; // this wave's part of dk, its first token tile
        const int h = hk * shared + hs;
        if (hs) {
            p = gdr_chunk(d, id / d.Hk, h);
            lds_barrier(); // everything in LDS of the head before is done with
        }
        const size_t gate = (p.tok + min(lane, rows - 1)) * d.H + h, val = (p.tok * d.H + h) * DV;
        float g = a.g[gate], be = a.beta[gate];
        if (lane >= rows) g = be = 0.f;
        GdrDecay dec;
        dec.sums(g, lane);
        if (w == 0) {
            s_hi[lane] = dec.hi;
            s_lo[lane] = dec.lo;
            s_be[lane] = be;
            s_eg[lane] = GdrDecay::pow2(dec.hi, dec.lo);
            s_ec[lane] = GdrDecay::pow2(lane_value(dec.hi, 63) - dec.hi, lane_value(dec.lo, 63) - dec.lo);
        }
        // state fragments [DV / KS][DK / 16], this wave's tiles 2 part, 2 part + 1
        const Frag *Sg = static_cast<const Frag *>(a.states) + p.blk * (DK * DV / E) + part * 128 + lane;
        const Frag *Dg = static_cast<const Frag *>(a.dstates) + p.blk * (DK * DV / E) + part * 128 + lane;
        // transposed: rows of dk (Gd::row of tiles 2 part, 2 part + 1), columns: token 16 (it0 + i) + r
        f32x4 m1[3], m2[3], dq[NI][2], dk[NI][2], wk[NI][2];
        zero_acc(m1);
        zero_acc(m2);
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) dq[i][u] = dk[i][u] = wk[i][u] = f32x4{0.f, 0.f, 0.f, 0.f};
        const unsigned pairs = kPairs[w];
        float trace = 0.f;
        auto fragments = [&](Frag &sf, Frag &df, int hv, int s, int u) {
            const size_t at = (size_t)((hv * S64 + s) * (DK / 16) + u) * 64;
            sf = Sg[at];
            df = Dg[at];
        };
        auto states = [&](Frag (&sf)[S64][2], Frag (&df)[S64][2], int hv) {
#pragma unroll
            for (int s = 0; s < EARLY; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u) fragments(sf[s][u], df[s][u], hv, s, u);
        };
#pragma unroll 1
        for (int hv = 0; hv < DV / 64; ++hv) {
            // In 16 bits asked for before the tiles, so that one wait covers both: 183 us for 200, [4, 4 096] tokens, 16 heads, d = 128
            Frag sf[S64][2], df[S64][2];
            states(sf, df, hv);
            if (hv) lds_barrier(); // the tiles before these are done with
            tile(TileV{}, s_e, static_cast<const T *>(a.e) + val + hv * 64, rsv);
            tile(TileV{}, s_do, static_cast<const T *>(a.dO) + val + hv * 64, rsv);
            tile(TileV{}, s_dv, static_cast<const T *>(a.dv) + val + hv * 64, rsv);
            wait_vm<0>();
            lds_barrier();
            // dO E^T, dV E^T
#pragma unroll
            for (int u = 0; u < 3; ++u) {
                const int ta = pairs >> (4 * u + 2) & 3, tb = pairs >> (4 * u) & 3;
                if (u < 2 || w < 2) {
#pragma unroll
                    for (int s = 0; s < S64; ++s) {
                        const Frag b = TileV::row_frag(s_e, 16 * tb + r, s, kg);
                        m1[u] = gd_mma<T>(TileV::row_frag(s_do, 16 * ta + r, s, kg), b, m1[u]);
                        m2[u] = gd_mma<T>(TileV::row_frag(s_dv, 16 * ta + r, s, kg), b, m2[u]);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0); // (phases mixed by the compiler need more registers than there are)
            // S dO^T, S dV^T, D E^T
#pragma unroll
            for (int s = 0; s < S64; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (s >= EARLY) fragments(sf[s][u], df[s][u], hv, s, u);
                    if (it0 == 0) trace += dot(sf[s][u], df[s][u]); // (once per part)
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        const int tok = 16 * (it0 + i) + r;
                        dq[i][u] = gd_mma<T>(sf[s][u], TileV::row_frag(s_do, tok, s, kg), dq[i][u]);
                        dk[i][u] = gd_mma<T>(sf[s][u], TileV::row_frag(s_dv, tok, s, kg), dk[i][u]);
                        wk[i][u] = gd_mma<T>(df[s][u], TileV::row_frag(s_e, tok, s, kg), wk[i][u]);
                    }
                }
        }
        trace = reduce64(trace);
        if (lane == 0) s_tr[w] = trace;
        // sums over the value heads before this one (SHARED)
        f32x4 *sum = static_cast<f32x4 *>(a.sums) + ((size_t)id * 4 + w) * ((NI * 4 + 6) * 64) + lane;
        // q.k and k.k of the same tiles; W1, W2 and the sums of Z
        f32x4 z1[3], z2[3];
        zero_acc(z1);
        zero_acc(z2);
#pragma unroll
        for (int u = 0; u < 3; ++u) {
            const int ta = pairs >> (4 * u + 2) & 3, tb = pairs >> (4 * u) & 3;
            if (u < 2 || w < 2) {
#pragma unroll
                for (int s = 0; s < SK; ++s) {
                    const Frag b = TileK::row_frag(s_k, 16 * tb + r, s, kg);
                    z1[u] = gd_mma<T>(TileK::row_frag(s_q, 16 * ta + r, s, kg), b, z1[u]);
                    z2[u] = gd_mma<T>(TileK::row_frag(s_k, 16 * ta + r, s, kg), b, z2[u]);
                }
            }
        }
        // (rows and columns of Z by tile: a tile's sums go to its own place, [other tile][token]; in a tile on the diagonal token i's place among the
        // rows is for the tile's pairs i' >= i > j)
#pragma unroll
        for (int u = 0; u < 3; ++u) {
            const int ta = pairs >> (4 * u + 2) & 3, tb = pairs >> (4 * u) & 3;
            if (u < 2 || w < 2) {
                const int j = 16 * tb + r;
                const float hj = s_hi[j], lj = s_lo[j], bj = s_be[j];
                f32x4 w1, w2, zb;
                float all = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int i = 16 * ta + 4 * kg + x;
                    const float c = GdrDecay::pow2(s_hi[i] - hj, s_lo[i] - lj);
                    const float v1 = i >= j && i < rows ? c * d.scale * m1[u][x] : 0.f, v2 = i > j && i < rows ? -c * m2[u][x] : 0.f;
                    const float z = v1 * z1[u][x] + v2 * z2[u][x];
                    w1[x] = bj * v1;
                    w2[x] = bj * v2;
                    all += z;
                    zb[x] = i > j ? bj * z : 0.f;
                }
                if (ta == tb) {
#pragma unroll
                    for (int x = 2; x >= 0; --x) zb[x] += zb[x + 1];
                    float from = zb[0]; // over the rows of this lane group and those behind it
                    const float x16 = __shfl_down(from, 16);
                    from += kg < 3 ? x16 : 0.f;
                    const float x32 = __shfl_down(from, 32);
                    from += kg < 2 ? x32 : 0.f;
                    const float next = __shfl_down(from, 16), behind = kg < 3 ? next : 0.f;
#pragma unroll
                    for (int x = 0; x < 4; ++x) zb[x] = r < 4 * kg + x ? zb[x] + behind : 0.f;
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float zr = reduce16(zb[x]);
                    if (r == 0) s_row[tb][16 * ta + 4 * kg + x] = zr;
                }
                all = add_xor32(add_xor16(all));
                if (kg == 0) s_col[ta][j] = all;
                if (SHARED && hs) {
                    w1 += sum[(NI * 4 + u) * 64];
                    w2 += sum[(NI * 4 + 3 + u) * 64];
                }
                if (SHARED && hs + 1 < shared) {
                    sum[(NI * 4 + u) * 64] = w1;
                    sum[(NI * 4 + 3 + u) * 64] = w2;
                } else {
                    store4(TileV::at(s_w1, j, 16 * ta + 4 * kg), w1);
                    store4(TileV::at(s_w2, j, 16 * ta + 4 * kg), w2);
                }
            } else if (u == 2) { // the tiles beside the diagonal that a 32-wide step reads
                const int j = 32 * (w - 2) + 16 + r, i = 32 * (w - 2) + 4 * kg;
                store4(TileV::at(s_w1, j, i), f32x4{0.f, 0.f, 0.f, 0.f});
                store4(TileV::at(s_w2, j, i), f32x4{0.f, 0.f, 0.f, 0.f});
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // what depends on the states alone: row dots a, b of this wave's part, scaled in place
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int tok = 16 * (it0 + i) + r;
            const float eg = s_eg[tok], ec = s_ec[tok], bt = s_be[tok];
            float av = 0.f, bv = 0.f;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int row0 = G::row(2 * part + u, 4 * kg);
                const f32x4 qv = load4(TileK::at(s_q, tok, row0)), kv = load4(TileK::at(s_k, tok, row0));
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    dq[i][u][x] *= eg * d.scale;
                    dk[i][u][x] *= -eg;
                    wk[i][u][x] *= ec;
                    av += qv[x] * dq[i][u][x] + kv[x] * dk[i][u][x];
                    bv += kv[x] * wk[i][u][x];
                    dk[i][u][x] += bt * wk[i][u][x];
                }
            }
            av = add_xor32(add_xor16(av));
            bv = add_xor32(add_xor16(bv));
            if (kg == 0) {
                s_a[part][tok] = av;
                s_b[part][tok] = bv;
            }
        }
        lds_barrier();
        if (w == 0) { // dg, dbeta: lane = token
            const int tile = lane >> 4;
            float all = s_b[0][lane], av = s_a[0][lane], bv = s_b[0][lane];
#pragma unroll
            for (int n = 1; n < NP; ++n) {
                av += s_a[n][lane];
                bv += s_b[n][lane];
                all += s_b[n][lane];
            }
            // pairs of this tile's rows and the tiles in front of it, of this tile's columns and the tiles behind it, of neither
            float rows_in = 0.f, cols_in = 0.f, to[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                to[n] = n > tile ? be * s_col[n][lane] : 0.f;
                cols_in += to[n];
                if (n < tile) rows_in += s_row[n][lane];
                if (n >= tile) all += s_col[n][lane];
            }
            const float t2 = reduce16(to[2]), t3 = reduce16(to[3]);
            const float across1 = lane_value(t2, 0) + lane_value(t3, 0), across2 = lane_value(t3, 0) + lane_value(t3, 16);
            const float across = tile == 1 ? across1 : tile == 2 ? across2 : 0.f;
            if (lane >= rows) av = bv = 0.f;
            // sums inside the tile: over the rows from this token on, over the columns in front of it
            rows_in += dpp_move<0x101>(rows_in); // row_shl 1, 2, 4, 8
            rows_in += dpp_move<0x102>(rows_in);
            rows_in += dpp_move<0x104>(rows_in);
            rows_in += dpp_move<0x108>(rows_in);
            cols_in = dpp_move<0x111>(cols_in); // row_shr 1; 1, 2, 4, 8
            cols_in += dpp_move<0x111>(cols_in);
            cols_in += dpp_move<0x112>(cols_in);
            cols_in += dpp_move<0x114>(cols_in);
            cols_in += dpp_move<0x118>(cols_in);
            const float pairs_here = s_row[tile][lane] + rows_in + cols_in + across;
            // sums over the tokens before this one, and over this one and those behind it
            float before = be * bv, behind = av;
#pragma unroll
            for (int n = 1; n < 64; n *= 2) {
                const float x = __shfl_up(before, n), y = __shfl_down(behind, n);
                before += lane >= n ? x : 0.f;
                behind += lane + n < 64 ? y : 0.f;
            }
            before = __shfl_up(before, 1);
            if (lane == 0) before = 0.f;
            float tr = s_tr[0];
#pragma unroll
            for (int n = 1; n < NP; ++n) tr += s_tr[n];
            if (lane < rows) {
                const float dg = pairs_here + before + behind + s_eg[63] * tr;
                if (sizeof(T) == 4 || a.f32_gates) {
                    static_cast<float *>(a.dg)[gate] = dg;
                    static_cast<float *>(a.dbeta)[gate] = all;
                } else {
                    static_cast<T *>(a.dg)[gate] = from_f32<T>(dg);
                    static_cast<T *>(a.dbeta)[gate] = from_f32<T>(all);
                }
            }
        }
        if (SHARED) {
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (hs) {
                        dq[i][u] += sum[(i * 4 + u) * 64];
                        dk[i][u] += sum[(i * 4 + 2 + u) * 64];
                    }
                    if (hs + 1 < shared) {
                        sum[(i * 4 + u) * 64] = dq[i][u];
                        sum[(i * 4 + 2 + u) * 64] = dk[i][u];
                    }
                }
            if (hs + 1 < shared) continue;
        }
        // dq += K^T W1^T, dk += K^T W2^T + Q^T W1 + K^T W2, all transposed
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < S64; ++s) {
                const Frag kf = TileK::col_frag(s_k, 2 * part + u, s, r, kg), qf = TileK::col_frag(s_q, 2 * part + u, s, r, kg);
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int it = it0 + i, tok = 16 * it + r;
                    if (s * G::KS < 16 * (it + 1)) { // tokens j of step s up to tile it
                        dq[i][u] = gd_mma<T>(kf, TileV::column_frag(s_w1, it, s, r, kg), dq[i][u]);
                        dk[i][u] = gd_mma<T>(kf, TileV::column_frag(s_w2, it, s, r, kg), dk[i][u]);
                    }
                    if ((s + 1) * G::KS > 16 * it) { // tokens i of step s from tile it on
                        dk[i][u] = gd_mma<T>(qf, TileV::row_frag(s_w1, tok, s, kg), dk[i][u]);
                        dk[i][u] = gd_mma<T>(kf, TileV::row_frag(s_w2, tok, s, kg), dk[i][u]);
                    }
                }
            }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int tok = 16 * (it0 + i) + r;
            if (tok < rows) {
                T *oq = static_cast<T *>(a.dq) + key + (size_t)tok * rsk, *ok = static_cast<T *>(a.dk) + key + (size_t)tok * rsk;
#pragma unroll
                for (int u = 0; u < 2; u += G::KT) {
                    const int c = G::row(2 * part + u, 4 * kg);
                    __builtin_nontemporal_store(G::frag(&dq[i][u]), reinterpret_cast<Frag *>(oq + c));
                    __builtin_nontemporal_store(G::frag(&dk[i][u]), reinterpret_cast<Frag *>(ok + c));
                }
            }
        }
    }
}

template <typename T, int DK, int DV> hipError_t launch(const GdrDims &d, const GdrGradArgs &a, hipStream_t s) {
    return launch_in_parts(d.nchunks * d.Hk, [&](int first, dim3 grid) {
        if (d.H > d.Hk) hipLaunchKernelGGL((gdr_grad_kernel<T, DK, DV, true>), grid, dim3(kThreads), 0, s, d, a, first);
        else hipLaunchKernelGGL((gdr_grad_kernel<T, DK, DV, false>), grid, dim3(kThreads), 0, s, d, a, first);
    });
}
template <typename T> hipError_t launch_t(const GdrDims &d, const GdrGradArgs &a, hipStream_t s) {
    if (d.dk == 64) return d.dv == 64 ? launch<T, 64, 64>(d, a, s) : launch<T, 64, 128>(d, a, s);
    return d.dv == 64 ? launch<T, 128, 64>(d, a, s) : launch<T, 128, 128>(d, a, s);
}

} // namespace

hipError_t launch_gdr_grad(const GdrDims &d, const GdrGradArgs &a, hipStream_t s) {
    return d.dtype == 1 ? launch_t<float>(d, a, s) : launch_t<bf16_t>(d, a, s);
}

} // namespace mdn
