// C-ABI front end of the operators beside the scan: argument validation on the
// host (before any HIP call), workspace layout, launches.
#include <limits.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "m3.h"
#include "m3_adamw.h"
#include "m3_ffn.h"
#include "m3_glr.h"
#include "m3_internal.h"

using namespace m3;

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
// Workgroups of one launch (a grid's threads are counted in 32 bits)
constexpr int64_t kMostGroups = INT64_C(1) << 22;
m3_status launched(hipError_t e) {
    if (e == hipSuccess) return M3_OK;
    note_hip_error(e);
    return M3_ERR_HIP;
}

// ---------------------------------------------------------------------------
// Gated linear recurrence
// ---------------------------------------------------------------------------

static_assert(glr::kChunk == M3_GLR_CHUNK, "chunk as documented");

// The token arrays' pointers: each on its element.  Channels a lane: two in
// bf16 where every row and pair of channels stays on four bytes, else one.
m3_status glr_vector(const m3_glr_dims *d, bool step, std::initializer_list<const void *> ptrs, bool z, int *V) {
    const uintptr_t e = d->io == M3_F32 ? 4 : 2;
    uintptr_t bits = 0;
    for (const void *p : ptrs) bits |= (uintptr_t)p;
    if (bits & (e - 1)) return M3_ERR_ALIGN;
    int64_t odd = d->width | d->x_stride_b | d->r_stride_b | d->i_stride_b | (z ? d->z_stride_b : 0);
    if (!step) odd |= d->x_stride_t | d->r_stride_t | d->i_stride_t | (z ? d->z_stride_t : 0);
    *V = (e == 2 && odd % 2 == 0 && (bits & 3) == 0) ? 2 : 1;
    return M3_OK;
}

m3_status check_glr(const m3_glr_dims *d, bool step) {
    if (!d) return M3_ERR_NULL;
    if (d->io != M3_F32 && d->io != M3_BF16) return M3_ERR_DTYPE;
    if (d->flags != 0 || d->batch < 1 || d->width < 1 || (!step && d->seqlen < 0)) return M3_ERR_SHAPE;
    const int64_t strides[] = {d->x_stride_b, d->x_stride_t, d->r_stride_b, d->r_stride_t,
                               d->i_stride_b, d->i_stride_t, d->z_stride_b, d->z_stride_t};
    // every element offset stays far inside 63 bits
    constexpr int64_t kMost = INT64_C(1) << 56;
    const int64_t L = step ? 1 : std::max<int64_t>(d->seqlen, 1);
    if (d->batch > INT_MAX || d->width > INT_MAX || d->batch * d->width > kMost / L) return M3_ERR_SHAPE;
    for (int64_t s : strides)
        if (s < 0 || s > kMost / std::max(L, d->batch)) return M3_ERR_SHAPE;
    // a workgroup's rows within 31-bit offsets
    for (int64_t s : {d->width, d->x_stride_t, d->r_stride_t, d->i_stride_t, d->z_stride_t})
        if (!step && s > (INT64_C(1) << 23)) return M3_ERR_SHAPE;
    if (step) return d->batch * d->width / 256 < kMostGroups ? M3_OK : M3_ERR_SHAPE;
    // one workgroup a tile (groups of 64 channels: the most)
    const int64_t tiles = (d->seqlen + glr::kChunk - 1) / glr::kChunk, groups = (d->width + 63) / 64;
    if (d->batch * groups > kMostGroups / std::max<int64_t>(tiles, 1)) return M3_ERR_SHAPE;
    return M3_OK;
}

struct GlrLayout {
    size_t inc, mapA, mapC, part, total;
};
GlrLayout glr_layout(const m3_glr_dims *d) {
    const size_t tiles = (size_t)((d->seqlen + glr::kChunk - 1) / glr::kChunk);
    const size_t words = round_up((size_t)d->batch * tiles * (size_t)d->width * sizeof(uint64_t), 256);
    GlrLayout w;
    w.inc = glr::kCtlBytes;
    w.mapA = w.inc + words;
    w.mapC = w.mapA + words;
    w.part = w.mapC + words;
    w.total = w.part + words;
    return w;
}

// Arguments that the forward and the backward share
template <class Args>
void glr_common(const m3_glr_dims *d, const void *x, const void *r, const void *i, const float *A, const void *z,
                int V, void *workspace, Args *a) {
    a->x = x; a->r = r; a->i = i; a->z = z; a->A = A;
    a->B = d->batch; a->L = d->seqlen; a->D = d->width;
    a->G = (d->width + 64 * V - 1) / (64 * V);
    a->tiles = (d->seqlen + glr::kChunk - 1) / glr::kChunk;
    a->x_sb = d->x_stride_b; a->x_st = d->x_stride_t; a->r_sb = d->r_stride_b; a->r_st = d->r_stride_t;
    a->i_sb = d->i_stride_b; a->i_st = d->i_stride_t; a->z_sb = d->z_stride_b; a->z_st = d->z_stride_t;
    const GlrLayout w = glr_layout(d);
    char *ws = static_cast<char *>(workspace);
    a->ctl = reinterpret_cast<uint64_t *>(ws);
    a->inc = reinterpret_cast<uint64_t *>(ws + w.inc);
    a->mapA = reinterpret_cast<uint64_t *>(ws + w.mapA);
    a->mapC = reinterpret_cast<uint64_t *>(ws + w.mapC);
    a->spin_max = wait_limit();
}

}  // namespace

extern "C" size_t m3_glr_workspace_bytes(const m3_glr_dims *d) {
    return check_glr(d, false) == M3_OK ? glr_layout(d).total : 0;
}

extern "C" m3_status m3_glr_fwd(const m3_glr_dims *d, const void *x, const void *r, const void *i, const float *A,
                                const void *z, const float *init_state, void *y, float *final_state, float *states,
                                void *workspace, size_t workspace_bytes, void *stream) {
    const m3_status s = check_glr(d, false);
    if (s != M3_OK) return s;
    if (!A || !final_state || (d->seqlen > 0 && (!x || !r || !i || !y))) return M3_ERR_NULL;
    int V = 1;
    const m3_status v = glr_vector(d, false, {x, r, i, z, y}, z != nullptr, &V);
    if (v != M3_OK) return v;
    for (const void *p : {(const void *)A, (const void *)init_state, (const void *)final_state, (const void *)states})
        if (!aligned(p, 4)) return M3_ERR_ALIGN;
    if (!aligned(workspace, 16)) return M3_ERR_ALIGN;
    if (!workspace || workspace_bytes < glr_layout(d).total) return M3_ERR_WORKSPACE;
    glr::FwdArgs a = {};
    glr_common(d, x, r, i, A, z, V, workspace, &a);
    a.init = init_state;
    a.y = y;
    a.final_state = final_state;
    a.states = states;
    return launched(glr::launch_fwd(a, d->io == M3_F32, V, static_cast<hipStream_t>(stream)));
}

extern "C" m3_status m3_glr_bwd(const m3_glr_dims *d, const void *x, const void *r, const void *i, const float *A,
                                const void *z, const float *states, const void *dy, const float *dfinal, void *dx,
                                void *dr, void *di, void *dz, float *dA, float *dinit_state, void *workspace,
                                size_t workspace_bytes, void *stream) {
    const m3_status s = check_glr(d, false);
    if (s != M3_OK) return s;
    if (!A || !dA || (d->seqlen > 0 && (!x || !r || !i || !states || !dy || !dx || !dr || !di || (z && !dz))))
        return M3_ERR_NULL;
    int V = 1;
    const m3_status v = glr_vector(d, false, {x, r, i, z, dy, dx, dr, di, dz}, z != nullptr, &V);
    if (v != M3_OK) return v;
    for (const void *p : {(const void *)A, (const void *)states, (const void *)dfinal, (const void *)dA,
                          (const void *)dinit_state})
        if (!aligned(p, 4)) return M3_ERR_ALIGN;
    if (!aligned(workspace, 16)) return M3_ERR_ALIGN;
    const GlrLayout w = glr_layout(d);
    if (!workspace || workspace_bytes < w.total) return M3_ERR_WORKSPACE;
    V = glr::bwd_channels(V, z != nullptr);
    glr::BwdArgs a = {};
    glr_common(d, x, r, i, A, z, V, workspace, &a);
    a.dy = dy; a.states = states; a.dfinal = dfinal;
    a.dx = dx; a.dr = dr; a.di = di; a.dz = dz; a.dA = dA; a.dinit = dinit_state;
    a.part = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + w.part);
    return launched(glr::launch_bwd(a, d->io == M3_F32, V, static_cast<hipStream_t>(stream)));
}

extern "C" m3_status m3_glr_step(const m3_glr_dims *d, float *state, const void *x, const void *r, const void *i,
                                 const float *A, const void *z, void *y, void *stream) {
    const m3_status s = check_glr(d, true);
    if (s != M3_OK) return s;
    if (!state || !x || !r || !i || !A || !y) return M3_ERR_NULL;
    int V = 1;
    const m3_status v = glr_vector(d, true, {x, r, i, z, y}, z != nullptr, &V);
    if (v != M3_OK) return v;
    if (!aligned(A, 4) || !aligned(state, 4)) return M3_ERR_ALIGN;
    glr::StepArgs a = {};
    a.state = state; a.x = x; a.r = r; a.i = i; a.z = z; a.A = A; a.y = y;
    a.B = d->batch; a.D = d->width;
    a.x_sb = d->x_stride_b; a.r_sb = d->r_stride_b; a.i_sb = d->i_stride_b; a.z_sb = d->z_stride_b;
    return launched(glr::launch_step(a, d->io == M3_F32, V, static_cast<hipStream_t>(stream)));
}

extern "C" m3_status m3_glr_check(const m3_glr_dims *d, const void *workspace, size_t workspace_bytes,
                                  uint32_t *timeouts, void *stream) {
    const m3_status s = check_glr(d, false);
    if (s != M3_OK) return s;
    if (!timeouts) return M3_ERR_NULL;
    if (!workspace || workspace_bytes < glr_layout(d).total) return M3_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return M3_ERR_ALIGN;
    if (d->seqlen <= glr::kChunk) {   // one tile a sequence: nothing waits
        *timeouts = 0;
        return M3_OK;
    }
    // ticket counter (the call count in its upper half), two timeout words
    uint32_t ctl[4];
    hipError_t e = hipMemcpyAsync(ctl, workspace, sizeof ctl, hipMemcpyDeviceToHost, static_cast<hipStream_t>(stream));
    if (e == hipSuccess) e = hipStreamSynchronize(static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return launched(e);
    *timeouts = ctl[2 + ((ctl[1] - 1u) & 1u)];
    return M3_OK;
}

// ---------------------------------------------------------------------------
// Gated feed-forward block
// ---------------------------------------------------------------------------

namespace {

m3_status check_ffn(const m3_ffn_dims *d, bool bwd) {
    if (!d) return M3_ERR_NULL;
    if (d->io != M3_F32 && d->io != M3_BF16) return M3_ERR_DTYPE;
    constexpr int64_t kMost = INT64_C(1) << 16;   // (a tile's rows stay within 31-bit offsets)
    if (d->tokens < 0 || d->dmodel < 1 || d->dff < 1 || d->dmodel > kMost || d->dff > kMost) return M3_ERR_SHAPE;
    if (d->tokens > (INT64_C(1) << 40) / std::max(d->dmodel, d->dff)) return M3_ERR_SHAPE;
    if (d->act != M3_ACT_SILU && d->act != M3_ACT_GELU) return M3_ERR_SHAPE;
    if (d->x_stride < d->dmodel || d->x_stride > 16 * kMost) return M3_ERR_SHAPE;
    if (bwd && (d->dy_stride < d->dmodel || d->dy_stride > 16 * kMost)) return M3_ERR_SHAPE;
    // the smallest tiles, 64 rows by 32 columns of a gate, in one launch
    const int64_t rows = std::max(d->tokens, std::max(d->dmodel, d->dff)) / 64 + 1;
    if (rows > kMostGroups / (std::max(d->dmodel, d->dff) / 32 + 1)) return M3_ERR_SHAPE;
    return M3_OK;
}

// Rows in the workspace start on 16 bytes: their lengths are whole pieces.
struct FfnLayout {
    int64_t Dp, Fp;
    bool pad_d, pad_f;             // rows of dmodel, of dff, are no whole pieces
    int64_t some;                  // tokens the gates' backward takes at a time
    size_t x, dy, wg, wu, wd, h, dg, du, dh, part, total;
};
// any: room for copies of the weights wherever they start
FfnLayout ffn_layout(const m3_ffn_dims *d, bool bwd, bool any) {
    const int64_t e = d->io == M3_F32 ? 4 : 2, el = 16 / e;
    FfnLayout w = {};
    w.Dp = (d->dmodel + el - 1) / el * el;
    w.Fp = (d->dff + el - 1) / el * el;
    w.pad_d = w.Dp != d->dmodel;
    w.pad_f = w.Fp != d->dff;
    // Tokens whose dh, in tiles of 256, gives each of the 256 compute units one:
    // up to 64 MB of fp32, read again by the gates while the cache of 256 MB past
    // L2 has it.
    w.some = 256 * std::max<int64_t>(1, 256 / ((w.Fp + 255) / 256));
    size_t at = 0;
    auto take = [&](int64_t rows, int64_t cols, int64_t bytes) {
        const size_t here = at;
        at = round_up(at + (size_t)(rows * cols * bytes), 256);
        return here;
    };
    w.x = take(d->tokens, w.Dp, e);                       // (used where x's rows need it)
    w.dy = bwd ? take(d->tokens, w.Dp, e) : 0;
    w.wg = take(w.pad_d || any ? d->dff : 0, w.Dp, e);
    w.wu = take(w.pad_d || any ? d->dff : 0, w.Dp, e);
    w.wd = take(w.pad_f || any ? d->dmodel : 0, w.Fp, e);
    w.h = take(d->tokens, w.Fp, e);
    w.dg = bwd ? take(d->tokens, w.Fp, e) : 0;
    w.du = bwd ? take(d->tokens, w.Fp, e) : 0;
    w.dh = bwd ? take(std::min(d->tokens, w.some), w.Fp, 4) : 0;
    w.part = take(1, (int64_t)ffn::kPartBytes, 1);
    w.total = at;
    return w;
}

// An operand as the products take it
struct Rows {
    const void *p;
    int64_t ld;
};

struct Ffn {
    const m3_ffn_dims *d;
    FfnLayout w;
    char *ws;
    hipStream_t stream;
    bool f32;
    hipError_t e = hipSuccess;
    ffn::PadArgs pads = {};

    // (copied, where its rows need it, by the launch of copy())
    Rows whole(const void *p, int64_t ld, int64_t rows, int64_t cols, int64_t padded, size_t at) {
        const int64_t es = f32 ? 4 : 2;
        if (padded == cols && ld * es % 16 == 0 && aligned(p, 16)) return Rows{p, ld};
        if (rows > 0) pads.copy[pads.count++] = {p, ws + at, ld, padded, rows, cols};
        return Rows{ws + at, padded};
    }
    void copy() { e = ffn::launch_pad(pads, f32, stream); }
    void gemm(const ffn::GemmArgs &g, bool at, bool bt, ffn::Kind kind) {
        if (e == hipSuccess && g.M > 0 && g.N > 0) e = ffn::launch_gemm(g, f32, at, bt, kind, stream);
    }
    ffn::GemmArgs args(int64_t M, int64_t N, int64_t K, Rows a, Rows b, void *c, int64_t ldc) const {
        ffn::GemmArgs g = {};
        g.a[0] = g.a[1] = a.p; g.b[0] = g.b[1] = b.p;
        g.lda = a.ld; g.ldb = b.ld;
        g.M = M; g.N = N; g.K = K; g.nseg = g.batch = 1;
        g.part = reinterpret_cast<float *>(ws + w.part);
        g.c[0] = g.c[1] = c; g.ldc = ldc;
        g.gelu = d->act == M3_ACT_GELU;
        return g;
    }
};

}  // namespace

extern "C" size_t m3_ffn_workspace_bytes(const m3_ffn_dims *d, int what) {
    if (what & ~(M3_FFN_BACKWARD | M3_FFN_ANY_WEIGHTS)) return 0;
    const bool bwd = (what & M3_FFN_BACKWARD) != 0;
    return check_ffn(d, bwd) == M3_OK ? ffn_layout(d, bwd, (what & M3_FFN_ANY_WEIGHTS) != 0).total : 0;
}

// The layout too: with room for copies where whole rows of weights need them
static m3_status check_ffn_args(const m3_ffn_dims *d, bool bwd, const void *Wg, const void *Wu, const void *Wd,
                                std::initializer_list<const void *> rest, const void *workspace, size_t workspace_bytes,
                                FfnLayout *w) {
    if (!Wg || !Wu || !Wd) return M3_ERR_NULL;
    const uintptr_t e = d->io == M3_F32 ? 4 : 2;
    for (const void *p : {Wg, Wu, Wd})
        if (!aligned(p, e)) return M3_ERR_ALIGN;
    for (const void *p : rest)
        if (!aligned(p, e)) return M3_ERR_ALIGN;
    *w = ffn_layout(d, bwd, false);
    const bool any = (!w->pad_d && !(aligned(Wg, 16) && aligned(Wu, 16))) || (!w->pad_f && !aligned(Wd, 16));
    if (any) *w = ffn_layout(d, bwd, true);
    if (!workspace) return M3_ERR_WORKSPACE;
    if (workspace_bytes < w->total) return any ? M3_ERR_ALIGN : M3_ERR_WORKSPACE;
    return aligned(workspace, 16) ? M3_OK : M3_ERR_ALIGN;
}

extern "C" m3_status m3_ffn_fwd(const m3_ffn_dims *d, const void *x, const void *Wg, const void *Wu, const void *Wd,
                                void *y, void *workspace, size_t workspace_bytes, void *stream) {
    m3_status s = check_ffn(d, false);
    if (s != M3_OK) return s;
    FfnLayout w;
    if (d->tokens > 0 && (!x || !y)) return M3_ERR_NULL;
    s = check_ffn_args(d, false, Wg, Wu, Wd, {x, y}, workspace, workspace_bytes, &w);
    if (s != M3_OK || d->tokens == 0) return s;
    const int64_t T = d->tokens, D = d->dmodel, F = d->dff;
    Ffn f{d, w, static_cast<char *>(workspace), static_cast<hipStream_t>(stream), d->io == M3_F32};
    const Rows rx = f.whole(x, d->x_stride, T, D, w.Dp, w.x);
    const Rows rg = f.whole(Wg, D, F, D, w.Dp, w.wg), ru = f.whole(Wu, D, F, D, w.Dp, w.wu);
    const Rows rd = f.whole(Wd, F, D, F, w.Fp, w.wd), h{f.ws + w.h, w.Fp};
    f.copy();
    if (T <= ffn::kFewRows && f.e == hipSuccess) {
        // (K in whole pieces: the copies are padded with zeros, and so is h)
        ffn::FewArgs a = {rx.p, {rg.p, ru.p}, rx.ld, rg.ld, T, F, w.Dp, w.Fp, f.ws + w.h, w.Fp, d->act == M3_ACT_GELU, nullptr, 0, 0};
        f.e = ffn::launch_few(a, f.f32, true, f.stream);
        a = ffn::FewArgs{h.p, {rd.p, rd.p}, h.ld, rd.ld, T, D, w.Fp, D, y, D, 0, reinterpret_cast<float *>(f.ws + w.part), 0, 0};
        if (f.e == hipSuccess) f.e = ffn::launch_few(a, f.f32, false, f.stream);
        return launched(f.e);
    }
    ffn::GemmArgs g = f.args(T, F, D, rx, rg, f.ws + w.h, w.Fp);
    g.b[1] = ru.p;
    f.gemm(g, false, false, ffn::kGate);
    f.gemm(f.args(T, D, F, h, rd, y, D), false, false, ffn::kStore);
    return launched(f.e);
}

extern "C" m3_status m3_ffn_bwd(const m3_ffn_dims *d, const void *x, const void *Wg, const void *Wu, const void *Wd,
                                const void *dy, void *dx, void *dWg, void *dWu, void *dWd, void *workspace,
                                size_t workspace_bytes, void *stream) {
    m3_status s = check_ffn(d, true);
    if (s != M3_OK) return s;
    FfnLayout w;
    if (!dWg || !dWu || !dWd || (d->tokens > 0 && (!x || !dy || !dx))) return M3_ERR_NULL;
    s = check_ffn_args(d, true, Wg, Wu, Wd, {x, dy, dx, dWg, dWu, dWd}, workspace, workspace_bytes, &w);
    if (s != M3_OK) return s;
    const int64_t T = d->tokens, D = d->dmodel, F = d->dff;
    Ffn f{d, w, static_cast<char *>(workspace), static_cast<hipStream_t>(stream), d->io == M3_F32};
    const Rows rx = f.whole(x, d->x_stride, T, D, w.Dp, w.x), ry = f.whole(dy, d->dy_stride, T, D, w.Dp, w.dy);
    const Rows rg = f.whole(Wg, D, F, D, w.Dp, w.wg), ru = f.whole(Wu, D, F, D, w.Dp, w.wu);
    const Rows rd = f.whole(Wd, F, D, F, w.Fp, w.wd);
    f.copy();
    const Rows h{f.ws + w.h, w.Fp}, dg{f.ws + w.dg, w.Fp}, du{f.ws + w.du, w.Fp};
    const int64_t e = d->io == M3_F32 ? 4 : 2;
    auto from = [e](Rows r, int64_t t) { return Rows{static_cast<const char *>(r.p) + t * r.ld * e, r.ld}; };
    ffn::GemmArgs g;
    for (int64_t t = 0; t < T; t += w.some) {
        const int64_t n = std::min(w.some, T - t), at = t * w.Fp * e;
        // dh = dy Wd (with the padding's columns, zero, too)
        g = f.args(n, w.Fp, D, from(ry, t), rd, f.ws + w.dh, w.Fp);
        g.f32_out = 1;
        f.gemm(g, false, true, ffn::kStore);
        // g and u again; h, dg, du
        g = f.args(n, F, D, from(rx, t), rg, f.ws + w.h + at, w.Fp);
        g.b[1] = ru.p;
        g.dg = f.ws + w.dg + at; g.du = f.ws + w.du + at;
        g.dh = reinterpret_cast<const float *>(f.ws + w.dh);
        f.gemm(g, false, false, ffn::kGateBwd);
    }
    // dx = dg Wg + du Wu
    g = f.args(T, D, F, dg, rg, dx, D);
    g.a[1] = du.p; g.b[1] = ru.p; g.nseg = 2;
    f.gemm(g, false, true, ffn::kStore);
    // dWg = dg^T x, dWu = du^T x, dWd = dy^T h
    g = f.args(F, D, T, dg, rx, dWg, D);
    g.a[1] = du.p; g.c[1] = dWu;
    g.a[2] = ry.p; g.b[2] = h.p; g.c[2] = dWd;
    g.lda3 = ry.ld; g.ldb3 = h.ld; g.ldc3 = F;
    g.batch = 3;
    f.gemm(g, true, true, ffn::kStore);
    return launched(f.e);
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------

// Where a table's Now is
static size_t now_at(int64_t rows, int64_t groups) {
    return round_up((size_t)rows * sizeof(adamw::Tensor) + (size_t)groups * sizeof(int32_t), 16);
}

extern "C" m3_status m3_adamw_plan_make(const m3_adamw_tensor *tensors, int64_t count, int32_t grad_dtype, int32_t flags,
                                        m3_adamw_plan *plan, void *host_table, size_t table_bytes) {
    if (!plan || (count > 0 && !tensors)) return M3_ERR_NULL;
    if (grad_dtype != M3_F32 && grad_dtype != M3_BF16) return M3_ERR_DTYPE;
    if (count < 0 || count > INT_MAX || (flags & ~M3_ADAMW_8BIT)) return M3_ERR_SHAPE;
    const bool eight = (flags & M3_ADAMW_8BIT) != 0, gf32 = grad_dtype == M3_F32;
    int64_t rows = 0, groups = 0;
    for (int64_t k = 0; k < count; ++k) {
        const m3_adamw_tensor &t = tensors[k];
        if (t.n < 0 || !std::isfinite(t.decay)) return M3_ERR_SHAPE;
        if (t.n == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v || (eight && !t.scales)) return M3_ERR_NULL;
        if (!aligned(t.p, 4) || !aligned(t.g, gf32 ? 4 : 2) || !aligned(t.low, 2) || (eight && !aligned(t.scales, 4)) ||
            (!eight && (!aligned(t.m, 4) || !aligned(t.v, 4))))
            return M3_ERR_ALIGN;
        if (t.n / adamw::kChunkElems >= 2 * kMostGroups) return M3_ERR_SHAPE;
        groups += (t.n + adamw::kChunkElems - 1) / adamw::kChunkElems;
        if (groups > 2 * kMostGroups) return M3_ERR_SHAPE;
        ++rows;
    }
    const size_t head = (size_t)rows * sizeof(adamw::Tensor), bytes = now_at(rows, groups) + sizeof(adamw::Now);
    if (host_table) {
        if (table_bytes < bytes) return M3_ERR_WORKSPACE;
        if (!aligned(host_table, 8)) return M3_ERR_ALIGN;
        adamw::Tensor *row = static_cast<adamw::Tensor *>(host_table);
        int32_t *of = reinterpret_cast<int32_t *>(static_cast<char *>(host_table) + head), first = 0;
        for (int64_t k = 0, r = 0; k < count; ++k) {
            const m3_adamw_tensor &t = tensors[k];
            if (t.n == 0) continue;
            const int32_t chunks = (int32_t)((t.n + adamw::kChunkElems - 1) / adamw::kChunkElems);
            row[r] = adamw::Tensor{t.p, t.g, t.m, t.v, t.low, t.scales, first, chunks,
                                   (int32_t)(t.n - (int64_t)(chunks - 1) * adamw::kChunkElems), (uint32_t)k, t.decay};
            std::fill(of + first, of + first + chunks, (int32_t)r);
            first += chunks;
            ++r;
        }
    }
    *plan = m3_adamw_plan{rows, groups, bytes, grad_dtype, flags};
    return M3_OK;
}

extern "C" m3_status m3_adamw_step(const m3_adamw_config *c, const m3_adamw_plan *plan, void *table,
                                   const float *grad_scale, void *stream) {
    if (!c || !plan || (plan->groups > 0 && !table)) return M3_ERR_NULL;
    if (plan->grad_dtype != M3_F32 && plan->grad_dtype != M3_BF16) return M3_ERR_DTYPE;
    if (plan->rows < 0 || plan->rows > plan->groups || plan->groups > 2 * kMostGroups || (plan->flags & ~M3_ADAMW_8BIT) ||
        (!c->device_step && c->step < 1))
        return M3_ERR_SHAPE;
    if ((!c->device_lr && !std::isfinite(c->lr)) || !(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0) ||
        !(c->eps >= 0.0) || !std::isfinite(c->eps))
        return M3_ERR_SHAPE;
    if (!aligned(grad_scale, 4) || !aligned(table, 16) || !aligned(c->device_step, 8) || !aligned(c->device_lr, 8)) return M3_ERR_ALIGN;
    if (plan->groups == 0) return M3_OK;
    adamw::Args a = {};
    a.t = static_cast<const adamw::Tensor *>(table);
    a.of = reinterpret_cast<const int32_t *>(a.t + plan->rows);
    a.groups = (int32_t)plan->groups;
    a.b1 = (float)c->beta1; a.c1 = (float)(1.0 - c->beta1);
    a.b2 = (float)c->beta2; a.c2 = (float)(1.0 - c->beta2);
    a.eps = (float)c->eps;
    a.grad_scale = grad_scale;
    if (c->device_step || c->device_lr) {
        adamw::Now *now = reinterpret_cast<adamw::Now *>(static_cast<char *>(table) + now_at(plan->rows, plan->groups));
        a.from = now;
        const hipError_t e = adamw::launch_now(adamw::NowArgs{now, c->lr, c->beta1, c->beta2, c->step, c->seed, c->device_step, c->device_lr},
                                               static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return launched(e);
    } else {
        a.now = adamw::now(c->lr, c->beta1, c->beta2, c->step, c->seed);
    }
    return launched(adamw::launch(a, plan->grad_dtype == M3_F32, (plan->flags & M3_ADAMW_8BIT) != 0, static_cast<hipStream_t>(stream)));
}
