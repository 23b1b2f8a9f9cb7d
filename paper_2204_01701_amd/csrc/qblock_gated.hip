// qblock_gated.hip -- host side of the gated layer of include/qblock.h.
#include <cmath>

#include "qblock_gated.h"
#include "qblock_host.h"

using namespace ql;
using namespace ql::host;

namespace {

constexpr int kMostGated = 1 << 19;  // (256 rows of 2 n floats lie within a buffer resource)

bool gated_ok(const qblock_gated_desc *d) {
    return d && d->m >= 0 && d->k > 0 && d->n > 0 && float_type(d->dtype) && known_act(d->act) && d->ldx >= d->k && d->ldw >= d->k;
}
bool sizes_fit(const qblock_gated_desc *d) { return d->m <= kMostInt && d->k <= kMostGated && d->n <= kMostGated; }

int vec(ql_dtype t) { return t == QL_BF16 ? 8 : 4; }
int step_of(ql_dtype t) { return 64 / (int)esize(t); }
int whole_vectors(const qblock_gated_desc *d) { return (d->k + vec(d->dtype) - 1) / vec(d->dtype) * vec(d->dtype); }
int half_columns(const qblock_gated_desc *d) { return cdiv(d->n, step_of(d->dtype)) * step_of(d->dtype); }

// Rows of k elements that lie ld apart: whole aligned vectors, a tile's offsets within a buffer resource.
bool direct(const qblock_gated_desc *d, long long ld) {
    return d->k % vec(d->dtype) == 0 && ld % vec(d->dtype) == 0 && !d->unaligned && (double)ld * (double)esize(d->dtype) * 256 < 2147483648.0;
}

enum Tile { TILE_64, TILE_128, TILE_256 };  // 64 x 128, 128 x 128, 256 x 256 of C
int tile_rows(Tile t) { return t == TILE_256 ? 256 : t == TILE_128 ? 128 : 64; }
int tile_cols(Tile t) { return t == TILE_256 ? 256 : 128; }
int tile_threads(Tile t) { return t == TILE_256 ? 512 : 256; }

struct GatedPlan {
    Tile tile;
    int ti, tj, steps, splits, per;
    size_t part_bytes;
    double us;
};

// Time of a product in us by tile and splits: rounds of the workgroups over the CUs, each with its ramp and epilogue;
// per K step kStepUs; the partial sums go out and come back at 4.5 TB/s, and joining them is a launch (the form and the
// steps' times of the first-order layer's model, whose main loop this is).
constexpr double kStepUs[2][3] = {{0.54, 1.03, 3.66}, {0.20, 0.30, 0.86}};  // fp32, bf16
GatedPlan plan(GatedMode mode, const qblock_gated_desc *d) {
    const bool bf16 = d->dtype == QL_BF16;
    const int bk = step_of(d->dtype);
    const long long rows = mode == GATED_DW ? d->n : d->m, cols = mode == GATED_FWD ? 2LL * d->n : d->k;
    const double size = (mode == GATED_DW ? 2.0 : 1.0) * (double)rows * cols;
    GatedPlan p{};
    p.steps = mode == GATED_FWD ? cdiv(d->k, bk) : mode == GATED_DX ? 2 * (half_columns(d) / bk) : cdiv(d->m, bk);
    const int forced = env_override("QBLOCK_TILE", -1), forced_splits = env_override("QBLOCK_SPLITS", 0);
    double best = 1e300;
    int want = 1;
    for (Tile t : {TILE_64, TILE_128, TILE_256}) {
        if (forced >= 0 && (int)t != forced) continue;
        const int ti = cdiv(rows, tile_rows(t)) * (mode == GATED_DW ? 2 : 1);
        const int tj = mode == GATED_FWD ? cdiv(d->n, tile_cols(t) / 2) : cdiv(cols, tile_cols(t));
        for (int s = 1; s == 1 || (s <= 16 && 4 * s <= p.steps && 4.0 * s * size <= (double)kMaxSplitBytes); ++s) {
            if (forced_splits && s != std::min(forced_splits, std::max(1, p.steps / 4))) continue;
            const double wgs = (double)ti * tj * s;
            if (wgs * tile_threads(t) >= 4294967296.0) continue;
            const double join = s > 1 ? 3.5 + 8.0 * s * size / 4.5e6 : 0.0;
            const double c = (t == TILE_256 ? 8.0 : 5.0) + kStepUs[bf16][t] * cdiv(p.steps, s) * std::ceil(wgs / kNumCUs) + join;
            if (c < best) best = c, want = s, p.tile = t, p.ti = ti, p.tj = tj;
        }
    }
    p.us = best;
    p.per = std::max(1, cdiv(p.steps, want));
    p.splits = std::max(1, cdiv(p.steps, p.per));
    if (p.splits > 1) p.part_bytes = align_up((size_t)p.splits * (size_t)size * sizeof(float));
    return p;
}

// Steps until the last CU is done with n1 tiles of s1 steps and then n2 of s2 <= s1, each taken by the first CU that is free.
long long makespan(long long n1, int s1, long long n2, int s2) {
    const long long low = n1 / kNumCUs * s1, high = n1 % kNumCUs ? low + s1 : low, behind = n1 % kNumCUs;
    long long a = high, b = high + (n2 / kNumCUs + 1) * s2;
    while (a < b) {
        const long long m = (a + b) / 2, fits = (kNumCUs - behind) * ((m - low) / s2) + behind * ((m - high) / s2);
        if (fits >= n2) b = m;
        else a = m + 1;
    }
    return a;
}

// The backward's products: one after the other, or in one launch of the same tiles without splits.
struct GradsPlan {
    bool both;
    GatedPlan dx, dw;
};
GradsPlan plan_grads(const qblock_gated_desc *d) {
    GradsPlan p{false, plan(GATED_DX, d), plan(GATED_DW, d)};
    const int forced = env_override("QBLOCK_BOTH", -1), forced_tile = env_override("QBLOCK_TILE", -1);
    if (forced == 0 || d->m == 0) return p;
    const int bk = step_of(d->dtype);
    double best = forced == 1 ? 1e300 : p.dx.us + p.dw.us;
    for (Tile t : {TILE_64, TILE_128, TILE_256}) {
        if (forced_tile >= 0 && (int)t != forced_tile) continue;
        // (bf16 in the large tiles, of which a CU holds one, is what the sum of steps describes: 526 us for 4096 x 2048 -> 8192,
        // in turn 554.  Small tiles share a CU; of float32 one size was measured, 2048 x 1024 -> 4096 of many tiles: 660 us in one
        // launch, in turn 558.  Sizes with fewer tiles than CUs were not)
        if (forced != 1 && (t != TILE_256 || d->dtype != QL_BF16)) continue;
        GatedPlan x{}, w{};
        x.tile = w.tile = t;
        x.splits = w.splits = 1;
        x.ti = cdiv(d->m, tile_rows(t)), x.tj = cdiv(d->k, tile_cols(t));
        w.ti = 2 * cdiv(d->n, tile_rows(t)), w.tj = cdiv(d->k, tile_cols(t));
        x.per = x.steps = 2 * (half_columns(d) / bk);
        w.per = w.steps = cdiv(d->m, bk);
        const long long nx = (long long)x.ti * x.tj, nw = (long long)w.ti * w.tj;
        if ((double)(nx + nw) * tile_threads(t) >= 4294967296.0) continue;
        const long long m = x.steps >= w.steps ? makespan(nx, x.steps, nw, w.steps) : makespan(nw, w.steps, nx, x.steps);
        const double us = (t == TILE_256 ? 8.0 : 5.0) + kStepUs[d->dtype == QL_BF16][t] * (double)m;
        if (us < best) best = us, p = GradsPlan{true, x, w};
    }
    return p;
}

// (1 row of 4096 -> 8192 takes 32 us in bf16 and 62 in float32, 16 rows 37 and 63.  In bf16 the tiles, which take 28 for 64 rows, may be
// faster from a few rows on; they need a workspace for splits and whole vectors)
bool few_rows(const qblock_gated_desc *d, bool keep) { return d->m <= QBLOCK_FEW_ROWS && !keep; }

struct Pads {
    size_t x, w;  // bytes of x's copy, of one weight's
    Pads(const qblock_gated_desc *d, bool need_x, bool need_w) {
        const size_t row = (size_t)whole_vectors(d) * esize(d->dtype);
        x = need_x && !direct(d, d->ldx) ? align_up((size_t)d->m * row) : 0;
        w = need_w && !direct(d, d->ldw) ? align_up((size_t)d->n * row) : 0;
    }
};

// Rows of k elements -> rows of whole vectors at `to`.
template <typename T> const void *pad(const qblock_gated_desc *d, const void *p, long long ld, long long rows, void *to, hipStream_t st) {
    const int cols = whole_vectors(d);
    hipLaunchKernelGGL((qhead_pad_kernel<T>), dim3(grid_1d(rows * (cols / vec(d->dtype)))), dim3(kThreads), 0, st,
                       static_cast<const T *>(p), ld, rows, d->k, cols, static_cast<T *>(to));
    return to;
}

template <typename T, int MODE> ql_status launch(const GatedPlan &p, GatedArgs a, hipStream_t st) {
    a.ti = p.ti, a.tj = p.tj, a.splits = p.splits, a.per = p.per, a.steps = p.steps;
    const dim3 grid((unsigned)((long long)p.ti * p.tj * p.splits));
    if (p.tile == TILE_256) hipLaunchKernelGGL((qblock_gated_kernel<T, MODE, 256, 256, 2, 4, 4, 1, 2>), grid, dim3(512), 0, st, a);
    else if (p.tile == TILE_128) hipLaunchKernelGGL((qblock_gated_kernel<T, MODE, 128, 128, 2, 2, 4, 2, 4>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((qblock_gated_kernel<T, MODE, 64, 128, 2, 2, 4, 2, 3>), grid, dim3(256), 0, st, a);
    if (p.splits > 1) {
        const long long rows = MODE == GATED_DW ? 2LL * a.I : a.I;
        hipLaunchKernelGGL((qblock_gated_join_kernel<T, MODE>), dim3(grid_1d(rows * cdiv(a.J, kKeep) * 4)), dim3(kThreads), 0, st, a);
    }
    return hip_status();
}

template <typename T> ql_status launch_both(const GradsPlan &p, GatedArgs dx, GatedArgs dw, hipStream_t st) {
    for (auto *q : {&dx, &dw}) {
        const GatedPlan &g = q == &dx ? p.dx : p.dw;
        q->ti = g.ti, q->tj = g.tj, q->splits = 1, q->per = g.per, q->steps = g.steps;
    }
    const int nx = p.dx.ti * p.dx.tj, nw = p.dw.ti * p.dw.tj;
    const bool dx_first = p.dx.steps >= p.dw.steps;
    const int dx0 = dx_first ? 0 : nw, dw0 = dx_first ? nx : 0;
    const dim3 grid((unsigned)(nx + nw));
    if (p.dx.tile == TILE_256) hipLaunchKernelGGL((qblock_gated_grads_kernel<T, 256, 256, 2, 4, 4, 1, 2>), grid, dim3(512), 0, st, dx, dw, dx0, dw0);
    else if (p.dx.tile == TILE_128) hipLaunchKernelGGL((qblock_gated_grads_kernel<T, 128, 128, 2, 2, 4, 2, 4>), grid, dim3(256), 0, st, dx, dw, dx0, dw0);
    else hipLaunchKernelGGL((qblock_gated_grads_kernel<T, 64, 128, 2, 2, 4, 2, 3>), grid, dim3(256), 0, st, dx, dw, dx0, dw0);
    return hip_status();
}

bool pointers_fit(const qblock_gated_desc *d, const void *x, const void *wg, const void *wu) {
    return d->unaligned || (aligned16(x) && aligned16(wg) && aligned16(wu)) || d->k % vec(d->dtype) != 0;
}

template <typename T>
ql_status forward(const qblock_gated_desc *d, const void *x, const void *wg, const void *wu, const GatedOut &o, char *ws, hipStream_t st) {
    GatedArgs a{};
    a.a = x, a.b0 = wg, a.b1 = wu, a.lda = d->ldx, a.ldb = d->ldw;
    a.I = d->m, a.J = d->n, a.R = d->k, a.o = o;
    if (few_rows(d, o.q != nullptr)) {
        hipLaunchKernelGGL((qblock_gated_few_kernel<T>), dim3(cdiv(d->n, 16)), dim3(512), 0, st, a);
        return hip_status();
    }
    const Pads pads(d, true, true);
    if (pads.x) a.a = pad<T>(d, x, d->ldx, d->m, ws, st), a.lda = whole_vectors(d);
    if (pads.w) {
        a.b0 = pad<T>(d, wg, d->ldw, d->n, ws + pads.x, st);
        a.b1 = pad<T>(d, wu, d->ldw, d->n, ws + pads.x + pads.w, st);
        a.ldb = whole_vectors(d);
    }
    a.part = reinterpret_cast<float *>(ws + pads.x + 2 * pads.w);
    return launch<T, GATED_FWD>(plan(GATED_FWD, d), a, st);
}

struct DzPlan {
    int rpp, parts;
    size_t dz_bytes, part_bytes;
    explicit DzPlan(const qblock_gated_desc *d) {
        // (up to 64 rows are one part, whose sums are the results themselves.  A part has at most 1024 rows, 128 a thread, as long as
        // a grid's 65535 rows of workgroups take the parts, up to 2^26 rows: 2^24 rows in 128 parts made sums of 16384 terms, whose
        // roundings added up to 3900 x 2^-24; a second sum in the kernel, for every 64 rows, gives the same bound and costs 1.5 % of every pass)
        rpp = d->m <= 64 ? std::max(1, d->m) : std::max({32, std::min(1024, cdiv(d->m, 128)), cdiv(d->m, 65535)});
        parts = std::max(1, cdiv(d->m, rpp));
        dz_bytes = align_up((size_t)d->m * 2 * half_columns(d) * esize(d->dtype));
        part_bytes = parts > 1 ? align_up((size_t)parts * 2 * d->n * sizeof(float)) : 0;
    }
};

template <typename T>
ql_status backward(const qblock_gated_desc *d, const void *x, const void *wg, const void *wu, const void *dh, const void *z, const int8_t *q,
                   const uint8_t *e, void *dx, void *dwg, void *dwu, float *dbg, float *dbu, char *ws, hipStream_t st) {
    const DzPlan p(d);
    const int np = half_columns(d);
    float *sums = reinterpret_cast<float *>(ws + p.dz_bytes);
    const bool joined = p.parts > 1;
    GatedDzArgs z0{dh, d->ldh, z, q, e, d->m, d->n, np, (int)d->act, p.rpp, dx || dwg ? ws : nullptr,
                   !dbg ? nullptr : joined ? sums : dbg, !dbu ? nullptr : joined ? sums + (size_t)p.parts * d->n : dbu, d->n};
    const dim3 grid(cdiv(np, 256), p.parts);
    if (z) hipLaunchKernelGGL((qblock_gated_dz_kernel<T, false>), grid, dim3(kThreads), 0, st, z0);
    else hipLaunchKernelGGL((qblock_gated_dz_kernel<T, true>), grid, dim3(kThreads), 0, st, z0);
    if (joined && (dbg || dbu))
        hipLaunchKernelGGL(qblock_gated_colsum_kernel<>, dim3(cdiv(d->n, 32), 2), dim3(kThreads), 0, st, z0.part0, z0.part1, p.parts, d->n, dbg, dbu);
    ql_status s = hip_status();
    if (s != QL_OK || (!dx && !dwg)) return s;
    GatedArgs x0{}, w0{};
    x0.a = w0.a = ws, x0.lda = w0.lda = 2LL * np, x0.np = w0.np = np;
    ws += p.dz_bytes + p.part_bytes;
    const GradsPlan plans = plan_grads(d);
    const bool both = plans.both && dx && dwg;
    const Pads pads(d, dwg != nullptr, dx != nullptr);
    if (dx) {
        x0.b0 = wg, x0.b1 = wu, x0.ldb = d->ldw;
        if (pads.w) {
            x0.b0 = pad<T>(d, wg, d->ldw, d->n, ws, st);
            x0.b1 = pad<T>(d, wu, d->ldw, d->n, ws + pads.w, st);
            x0.ldb = whole_vectors(d);
        }
        x0.I = d->m, x0.J = d->k, x0.R = d->n, x0.o.c0 = dx;
        x0.part = reinterpret_cast<float *>(ws + 2 * pads.w);
        if (!both) s = launch<T, GATED_DX>(plans.both ? plan(GATED_DX, d) : plans.dx, x0, st);
    }
    if (dwg && s == QL_OK) {
        if (both) ws += 2 * pads.w;  // (else the products run one after the other on the same piece)
        w0.b0 = w0.b1 = x, w0.ldb = d->ldx;
        if (pads.x) w0.b0 = w0.b1 = pad<T>(d, x, d->ldx, d->m, ws, st), w0.ldb = whole_vectors(d);
        w0.I = d->n, w0.J = d->k, w0.R = d->m, w0.o.c0 = dwg, w0.o.c1 = dwu, w0.o.c_f32 = d->dw_f32 != 0;
        w0.part = reinterpret_cast<float *>(ws + pads.x);
        s = both ? launch_both<T>(plans, x0, w0, st) : launch<T, GATED_DW>(plans.both ? plan(GATED_DW, d) : plans.dw, w0, st);
    }
    return s;
}

}  // namespace

extern "C" {

size_t qblock_gated_fwd_workspace_size(const qblock_gated_desc *d) {
    if (!gated_ok(d) || !sizes_fit(d) || d->m == 0) return 0;
    const Pads pads(d, true, true);  // (few rows without a checkpoint need nothing, with one they do)
    return pads.x + 2 * pads.w + plan(GATED_FWD, d).part_bytes;
}

ql_status qblock_gated_fwd(const qblock_gated_desc *d, const void *x, const void *wg, const void *wu, const float *bg, const float *bu,
                           void *h, void *z, int8_t *q, uint8_t *e, void *workspace, size_t workspace_bytes, void *stream) {
    if (!gated_ok(d) || d->ldh < d->n || !q != !e) return QL_EINVAL;
    if (!sizes_fit(d)) return QL_EUNSUPPORTED;
    if (d->m == 0) return QL_OK;
    if (!x || !wg || !wu || !h) return QL_EINVAL;
    const void *ptrs[] = {x, wg, wu, h, z};
    for (const void *p : ptrs)
        if (!aligned(p, esize(d->dtype))) return QL_EINVAL;
    if (!aligned(bg, 4) || !aligned(bu, 4)) return QL_EINVAL;
    if (!few_rows(d, q != nullptr)) {
        if (!pointers_fit(d, x, wg, wu)) return QL_EINVAL;
        const size_t need = qblock_gated_fwd_workspace_size(d);
        if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
        if (workspace && !aligned16(workspace)) return QL_EINVAL;
    }
    const GatedOut o{bg, bu, h, d->ldh, z, q, e, (int)d->act, nullptr, nullptr, false};
    char *ws = static_cast<char *>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return d->dtype == QL_BF16 ? forward<uint16_t>(d, x, wg, wu, o, ws, st) : forward<float>(d, x, wg, wu, o, ws, st);
}

size_t qblock_gated_bwd_workspace_size(const qblock_gated_desc *d) {
    if (!gated_ok(d) || !sizes_fit(d)) return 0;
    const DzPlan p(d);
    const Pads pads(d, true, true);
    // the two products run one after the other on the same piece, or in one launch (where both are asked for)
    size_t most = std::max(2 * pads.w + plan(GATED_DX, d).part_bytes, pads.x + plan(GATED_DW, d).part_bytes);
    if (plan_grads(d).both) most = std::max(most, pads.x + 2 * pads.w);
    return p.dz_bytes + p.part_bytes + most;
}

ql_status qblock_gated_bwd(const qblock_gated_desc *d, const void *x, const void *wg, const void *wu, const void *dh, const void *z,
                           const int8_t *q, const uint8_t *e, void *dx, void *dwg, void *dwu, float *dbg, float *dbu, void *workspace,
                           size_t workspace_bytes, void *stream) {
    if (!gated_ok(d) || d->ldh < d->n) return QL_EINVAL;
    if ((d->m > 0 && !dx && !dwg && !dbg && !dbu) || !dwg != !dwu) return QL_EINVAL;  // (of no rows dx is no pointer)
    if (!sizes_fit(d)) return QL_EUNSUPPORTED;
    if (d->m == 0) {
        if (!dwg && !dbg && !dbu) return QL_OK;
        dx = nullptr;  // (nothing to write there: a launch without workgroups, which HIP refuses, would end the call)
    }
    if (d->m > 0 && (!dh || (!z && (!q || !e)) || (dx && (!wg || !wu)) || (dwg && !x))) return QL_EINVAL;
    const void *ptrs[] = {x, wg, wu, dh, z, dx};
    for (const void *p : ptrs)
        if (!aligned(p, esize(d->dtype))) return QL_EINVAL;
    const size_t wa = d->dw_f32 ? 4 : esize(d->dtype);
    if (!aligned(dwg, wa) || !aligned(dwu, wa) || !aligned(dbg, 4) || !aligned(dbu, 4)) return QL_EINVAL;
    if (!pointers_fit(d, dwg ? x : nullptr, dx ? wg : nullptr, dx ? wu : nullptr)) return QL_EINVAL;
    const size_t need = qblock_gated_bwd_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    char *ws = static_cast<char *>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return d->dtype == QL_BF16 ? backward<uint16_t>(d, x, wg, wu, dh, z, q, e, dx, dwg, dwu, dbg, dbu, ws, st)
                               : backward<float>(d, x, wg, wu, dh, z, q, e, dx, dwg, dwu, dbg, dbu, ws, st);
}

}  // extern "C"
