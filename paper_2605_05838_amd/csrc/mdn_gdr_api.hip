// C ABI of the gated delta rule: argument checks, workspace carving, kernel sequencing.  The contract is in include/mdn.h.
#include "../../include/mdn.h"
#include "mdn_gdr.h"
#include "mdn_side.h"

#include <hip/hip_runtime.h>
#include <algorithm>
#include <mutex>
#include <new>
#include <vector>

using namespace mdn;

namespace {

struct Carve {
    char *base;
    size_t off = 0;
    explicit Carve(void *b) : base(static_cast<char *>(b)) {}
    template <typename P = void> P *take(size_t bytes) {
        char *p = base ? base + off : nullptr;
        off += (bytes + 255) / 256 * 256;
        return reinterpret_cast<P *>(p);
    }
};

int check_shape(const mdn_gdr_shape *s, GdrDims *d) {
    if (!s) return MDN_ERR_NULL;
    const int dtype = s->dtype & ~MDN_GDR_F32_GATE_GRADS;
    if (dtype != MDN_DTYPE_BF16 && dtype != MDN_DTYPE_F32) return MDN_ERR_DTYPE;
    if (s->B < 1 || s->T < 1 || s->H < 1 || s->Hk < 1 || s->H > 4096 || s->H % s->Hk) return MDN_ERR_SHAPE;
    if ((s->dk != 64 && s->dk != 128) || (s->dv != 64 && s->dv != 128)) return MDN_ERR_SHAPE;
    if ((long long)s->B * s->H > (1 << 24) || ((long long)s->B * s->T + 64) * s->H > (1LL << 31) - 1) return MDN_ERR_SHAPE;
    *d = GdrDims{};
    d->B = s->B; d->T = s->T; d->H = s->H; d->Hk = s->Hk;
    d->N = (int)(((long long)s->T + 63) / 64);
    d->cn = d->N;
    d->nchunks = (int)((long long)s->B * d->N);
    d->dk = s->dk; d->dv = s->dv; d->dtype = dtype; d->scale = s->scale;
    return MDN_OK;
}

// cu: null for sequences of equal lengths
int check(const mdn_gdr_shape *s, const int32_t *cu, int32_t n_seq, GdrDims *d) {
    const int rc = check_shape(s, d);
    if (rc) return rc;
    if (!cu) return n_seq ? MDN_ERR_NULL : MDN_OK;
    if (s->B != 1 || n_seq < 1 || (long long)n_seq * s->H > (1 << 24)) return MDN_ERR_SHAPE;
    if (cu[0] != 0 || cu[n_seq] != s->T) return MDN_ERR_SHAPE;
    long long chunks = 0, longest = 0;
    for (int i = 0; i < n_seq; ++i) {
        if (cu[i + 1] <= cu[i] || cu[i + 1] > s->T) return MDN_ERR_SHAPE;
        const long long n = ((long long)cu[i + 1] - cu[i] + 63) / 64;
        chunks += n;
        longest = std::max(longest, n);
    }
    d->B = n_seq;
    d->N = (int)longest;
    d->nchunks = (int)chunks;
    return MDN_OK;
}

size_t elem(const GdrDims &d) { return d.dtype == MDN_DTYPE_F32 ? 4 : 2; }
size_t blocks(const GdrDims &d) { return (size_t)d.nchunks * d.H; }
size_t states_bytes(const GdrDims &d) { return blocks(d) * d.dk * d.dv * elem(d); }

struct Tables { SeqEntry *seqs; ChunkEntry *chunks; };
Tables carve_tables(Carve &c, const GdrDims &d, bool packed) {
    Tables t = {};
    if (packed) {
        t.seqs = c.take<SeqEntry>((size_t)d.B * sizeof(SeqEntry));
        t.chunks = c.take<ChunkEntry>((size_t)d.nchunks * sizeof(ChunkEntry));
    }
    return t;
}
// from the host's offsets, which travel in kernel arguments
int build_tables(GdrDims *d, const Tables &t, const int32_t *cu, hipStream_t s) {
    if (!cu) return MDN_OK;
    std::vector<SeqEntry> e;
    try {
        e.resize(d->B);
    } catch (const std::bad_alloc &) {
        return MDN_ERR_LAUNCH;
    }
    int cb = 0;
    for (int i = 0; i < d->B; ++i) {
        e[i] = SeqEntry{cu[i], cu[i + 1] - cu[i], cb, i};
        cb += (int)(((long long)e[i].len + 63) / 64);
    }
    // the longest first: their scans are what the others run beside
    std::sort(e.begin(), e.end(), [](const SeqEntry &a, const SeqEntry &b) { return a.len != b.len ? a.len > b.len : a.t0 < b.t0; });
    SeqList l;
    l.H = d->H;
    for (l.first = 0; l.first < d->B; l.first += l.n) {
        l.n = std::min(d->B - l.first, kSeqsPerLaunch);
        std::copy(e.begin() + l.first, e.begin() + l.first + l.n, l.e);
        if (launch_seq_tables(l, t.seqs, t.chunks, s) != hipSuccess) return MDN_ERR_LAUNCH;
    }
    d->seqs = t.seqs;
    d->chunks = t.chunks;
    return MDN_OK;
}

struct FwdWs { Tables tables; float *coef; void *T, *T_lo, *P; size_t total; };
FwdWs carve_fwd(const GdrDims &d, bool packed, void *ws) {
    Carve c(ws);
    FwdWs w;
    const size_t tri = blocks(d) * gdr_triangle_bytes(d.dtype);
    w.tables = carve_tables(c, d, packed);
    w.coef = c.take<float>(blocks(d) * kGdrCoef * sizeof(float));
    w.T = c.take(tri);
    w.T_lo = d.dtype == MDN_DTYPE_BF16 ? c.take(tri) : nullptr;
    w.P = c.take(tri);
    w.total = c.off;
    return w;
}

struct Operands { float *coef; void *TT, *PT; size_t total; };
Operands carve_operands(const GdrDims &d, void *p) {
    Carve c(p);
    Operands w;
    const size_t tri = blocks(d) * gdr_triangle_bytes(d.dtype);
    w.coef = c.take<float>(blocks(d) * kGdrCoef * sizeof(float));
    w.TT = c.take(tri);
    w.PT = c.take(tri);
    w.total = c.off;
    return w;
}

struct BwdWs { Tables tables; Operands op; void *TT_lo, *PT_lo, *states, *dstates, *sums; float *carry; size_t total; };
BwdWs carve_bwd(const GdrDims &d, bool packed, void *ws) {
    Carve c(ws);
    BwdWs w;
    const size_t tri = blocks(d) * gdr_triangle_bytes(d.dtype);
    w.tables = carve_tables(c, d, packed);
    void *op = c.take(carve_operands(d, nullptr).total);
    w.op = carve_operands(d, op);
    w.TT_lo = d.dtype == MDN_DTYPE_BF16 ? c.take(tri) : nullptr;
    w.PT_lo = d.dtype == MDN_DTYPE_BF16 ? c.take(tri) : nullptr;
    w.states = c.take(states_bytes(d));
    w.dstates = c.take(states_bytes(d));
    w.sums = d.H > d.Hk ? c.take((size_t)d.nchunks * d.Hk * gdr_sums_bytes(d.dk)) : nullptr;
    w.carry = packed ? nullptr : c.take<float>((size_t)d.B * d.H * d.dk * d.dv * sizeof(float));
    w.total = c.off;
    return w;
}

// Segments of a backward call: with scan workgroups for at most half of the CUs, the gradient launch of one runs beside the reverse scan of the
// one before it (in time) on the library's second stream, and so does the states' reconstruction beside the first scans.  The adjoint crosses
// a boundary in 32 bits, as the scan carries it: results do not depend on the number.  (Packed sequences' scans run beside each other.)
// A boundary costs ~10 us and hides a gradient launch, 40 us per 1 024 chunk blocks of d = 128: a segment per 1 024, at most 4; where the states are
// reconstructed, which the gradient launches wait for, 2, but with remainders, whose scans take longer, as many.  Backward in us, 1 / 2 / 4 / 8
// segments, states kept; reconstructed; reconstructed, with dS0 (16 heads of 128 unless said):
//    4 096 tokens    119 /   130 /   145 /   184;     172 /   151 /   174 /   232;     212 /   212 /   220 /   234
//    8 192           236 /   232 /   233 /   264;     334 /   262 /   280 /   325;     418 /   390 /   372 /   406
//   16 384           472 /   428 /   410 /   438;     685 /   499 /   526 /   558;     868 /   743 /   706 /   716
//   32 768           931 /   822 /   766 /   767;   1 366 /   957 /   985 / 1 039;   1 770 / 1 446 / 1 346 / 1 333
//   32 768, 4 heads  686 /   679 /   680 /   716;     976 /   704 /   700 /   745;   1 289 / 1 060 / 1 049 / 1 087
//   65 536, d = 64 1 336 / 1 269 / 1 237 / 1 255;   2 021 / 1 598 / 1 555 / 1 618;   2 601 / 2 043 / 1 952 / 1 972
//    4 096, 8, fp32  363 /   351 /   374 /   444;     500 /   375 /   394 /   557;     501 /   426 /   400 /   557
int segments(const GdrDims &d, bool rebuild, bool precise) {
    if (d.seqs) return 1;
    long long k = requested_segments();
    if (k <= 0) {
        if (2LL * ((d.B * d.H + 7) / 8 * 8) * (d.dv / 16) > num_cus()) return 1;
        k = (long long)d.nchunks * d.H * d.dk * (d.dtype == MDN_DTYPE_F32 ? 4 : 1) / (128 * 1024);
        if (rebuild && !precise && k) k = 2;
        k = std::min({4LL, d.N / 32LL, k});
    }
    return (int)std::max(1LL, std::min({16LL, k, d.N / 4LL}));
}
GdrDims segment(const GdrDims &d, int i, int k) {
    GdrDims r = d;
    r.c0 = (int)((long long)d.N * i / k);
    r.cn = (int)((long long)d.N * (i + 1) / k) - r.c0;
    r.nchunks = d.B * r.cn;
    return r;
}

int status(hipError_t e) { return e == hipSuccess ? MDN_OK : MDN_ERR_LAUNCH; }

template <size_t N> int check_pointers(const void *const (&required)[N], std::initializer_list<const void *> optional) {
    for (const void *p : required)
        if (!p) return MDN_ERR_NULL;
    for (const void *p : required)
        if (reinterpret_cast<uintptr_t>(p) & 15u) return MDN_ERR_ALIGN;
    for (const void *p : optional)
        if (reinterpret_cast<uintptr_t>(p) & 15u) return MDN_ERR_ALIGN;
    return MDN_OK;
}

} // namespace

extern "C" {

int mdn_gdr_bytes(const mdn_gdr_shape *shape, const int32_t *cu_seqlens, int32_t n_seq, int which, size_t *bytes_out) {
    if (!bytes_out) return MDN_ERR_NULL;
    GdrDims d;
    const int rc = check(shape, cu_seqlens, n_seq, &d);
    if (rc) return rc;
    switch (which) {
    case MDN_GDR_WS_FWD: *bytes_out = carve_fwd(d, cu_seqlens != nullptr, nullptr).total; return MDN_OK;
    case MDN_GDR_WS_BWD: *bytes_out = carve_bwd(d, cu_seqlens != nullptr, nullptr).total; return MDN_OK;
    case MDN_GDR_STATES: *bytes_out = states_bytes(d); return MDN_OK;
    case MDN_GDR_OPERANDS: *bytes_out = carve_operands(d, nullptr).total; return MDN_OK;
    default: return MDN_ERR_SHAPE;
    }
}

int mdn_gdr_chunk_fwd(const mdn_gdr_shape *shape, const int32_t *cu_seqlens, int32_t n_seq, const void *q, const void *k, const void *v,
                      const float *g, const float *beta, const float *S0, void *o, float *S_final, void *e_saved, void *states_saved,
                      void *operands_saved, void *workspace, size_t workspace_bytes, void *stream) {
    GdrDims d;
    int rc = check(shape, cu_seqlens, n_seq, &d);
    if (rc) return rc;
    const void *const required[] = {q, k, v, g, beta, o, workspace};
    rc = check_pointers(required, {S0, S_final, e_saved, states_saved, operands_saved});
    if (rc) return rc;
    const FwdWs w = carve_fwd(d, cu_seqlens != nullptr, workspace);
    if (workspace_bytes < w.total) return MDN_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    rc = build_tables(&d, w.tables, cu_seqlens, s);
    if (rc) return rc;
    const bool precise = d.dtype == MDN_DTYPE_BF16 && S_final;
    GdrLocalArgs l = {};
    l.q = q; l.k = k; l.g = g; l.beta = beta;
    l.coef = w.coef; l.T = w.T; l.T_lo = precise ? w.T_lo : nullptr; l.P = w.P;
    if (operands_saved) {
        const Operands op = carve_operands(d, operands_saved);
        l.coef = op.coef; l.TT = op.TT; l.PT = op.PT;
    }
    rc = status(launch_gdr_local(d, l, s));
    if (rc) return rc;
    GdrScanFwdArgs a = {};
    a.q = q; a.k = k; a.v = v; a.coef = l.coef; a.T = l.T; a.T_lo = l.T_lo; a.P = l.P; a.S0 = S0;
    a.o = o; a.e = e_saved; a.states = states_saved; a.S_final = S_final;
    return status(launch_gdr_scan_fwd(d, a, precise, s));
}

int mdn_gdr_chunk_bwd(const mdn_gdr_shape *shape, const int32_t *cu_seqlens, int32_t n_seq, const void *q, const void *k, const float *g,
                      const float *beta, const float *S0, const void *e_saved, const void *states_saved, const void *operands_saved,
                      const void *dO, const float *dS_final, void *dq, void *dk, void *dv, void *dg, void *dbeta, float *dS0,
                      void *workspace, size_t workspace_bytes, void *stream) {
    GdrDims d;
    int rc = check(shape, cu_seqlens, n_seq, &d);
    if (rc) return rc;
    const void *const required[] = {q, k, g, beta, e_saved, dO, dq, dk, dv, dg, dbeta, workspace};
    rc = check_pointers(required, {S0, states_saved, operands_saved, dS_final, dS0});
    if (rc) return rc;
    const BwdWs w = carve_bwd(d, cu_seqlens != nullptr, workspace);
    if (workspace_bytes < w.total) return MDN_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    rc = build_tables(&d, w.tables, cu_seqlens, s);
    if (rc) return rc;
    const bool precise = d.dtype == MDN_DTYPE_BF16 && dS0;
    Operands op = w.op;
    if (operands_saved && !precise) { // (the forward's have no remainders)
        op = carve_operands(d, const_cast<void *>(operands_saved));
    } else {
        GdrLocalArgs l = {};
        l.q = q; l.k = k; l.g = g; l.beta = beta;
        l.coef = op.coef; l.TT = op.TT; l.PT = op.PT;
        if (precise) l.TT_lo = w.TT_lo, l.PT_lo = w.PT_lo;
        rc = status(launch_gdr_local(d, l, s));
        if (rc) return rc;
    }
    GdrScanFwdArgs a = {}; // the states' reconstruction, where they were not kept
    a.k = k; a.v = e_saved; a.coef = op.coef; a.S0 = S0; a.states = w.states;
    GdrScanBwdArgs b = {};
    b.q = q; b.k = k; b.dO = dO; b.coef = op.coef; b.TT = op.TT; b.PT = op.PT;
    if (precise) b.TT_lo = w.TT_lo, b.PT_lo = w.PT_lo;
    b.dS_final = dS_final; b.dv = dv; b.dstates = w.dstates; b.dS0 = dS0;
    GdrGradArgs c = {};
    c.q = q; c.k = k; c.e = e_saved; c.dO = dO; c.dv = dv; c.g = g; c.beta = beta; c.states = states_saved ? states_saved : w.states;
    c.dstates = w.dstates; c.sums = w.sums; c.dq = dq; c.dk = dk; c.dg = dg; c.dbeta = dbeta;
    c.f32_gates = shape->dtype & MDN_GDR_F32_GATE_GRADS;
    const int nseg = segments(d, !states_saved, precise);
    if (nseg == 1) {
        if (!states_saved) { // before anything is written over S0
            rc = status(launch_gdr_rebuild(d, a, s));
            if (rc) return rc;
        }
        rc = status(launch_gdr_scan_bwd(d, b, precise, s));
        if (rc) return rc;
        return status(launch_gdr_grad(d, c, s));
    }
    Side *sdev = side_device();
    if (!sdev) return MDN_ERR_LAUNCH;
    std::lock_guard<std::mutex> lock(sdev->mutex);
    Side *sd = side(nseg + 3);
    if (!sd) return MDN_ERR_LAUNCH;
    auto hand_over = [&](hipEvent_t e, hipStream_t from, hipStream_t to) {
        return hipEventRecord(e, from) == hipSuccess && hipStreamWaitEvent(to, e, 0) == hipSuccess ? MDN_OK : MDN_ERR_LAUNCH;
    };
    if (!states_saved) {
        rc = hand_over(sd->ev[nseg], s, sd->stream);
        if (rc) return rc;
        rc = status(launch_gdr_rebuild(d, a, sd->stream));
        if (hipEventRecord(sd->ev[nseg + 1], sd->stream) != hipSuccess) rc = MDN_ERR_LAUNCH;
    }
    for (int i = nseg - 1; i >= 0 && !rc; --i) { // the last one first
        const GdrDims di = segment(d, i, nseg);
        b.dS_final = i == nseg - 1 ? dS_final : w.carry;
        b.dS0 = i == 0 ? dS0 : w.carry;
        if (i == 0 && dS0 && !states_saved) { // it may be written over S0, which the reconstruction reads
            if (hipStreamWaitEvent(s, sd->ev[nseg + 1], 0) != hipSuccess) rc = MDN_ERR_LAUNCH;
            if (rc) break;
        }
        rc = status(launch_gdr_scan_bwd(di, b, precise, s));
        if (!rc) rc = hand_over(sd->ev[i], s, sd->stream);
        if (!rc) rc = status(launch_gdr_grad(di, c, sd->stream));
    }
    // the caller's stream waits for whatever went to the second stream, also when a launch failed on the way
    const int joined = hand_over(sd->ev[nseg + 2], sd->stream, s);
    return rc ? rc : joined;
}

int mdn_gdr_recurrent_step(const mdn_gdr_shape *shape, const void *q, const void *k, const void *v, const float *g, const float *beta,
                           float *S, void *o, void *stream) {
    GdrDims d;
    int rc = check_shape(shape, &d);
    if (rc) return rc;
    const void *const required[] = {q, k, v, g, beta, S, o};
    rc = check_pointers(required, {});
    if (rc) return rc;
    GdrStepArgs a = {q, k, v, g, beta, S, o};
    return status(launch_gdr_step(d, a, static_cast<hipStream_t>(stream)));
}

} // extern "C"
