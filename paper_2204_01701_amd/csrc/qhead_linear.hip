// qhead_linear.hip -- host side of the first-order layer of include/qhead.h.
#include <cmath>

#include "qhead.h"
#include "qhead_gemm.h"
#include "qhost.h"

using namespace ql;
using namespace ql::host;

namespace {

size_t esize(ql_dtype t) { return t == QL_BF16 ? 2 : 4; }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool linear_ok(const qhead_linear_desc *d) {
    return d && d->m >= 0 && d->k > 0 && d->n > 0 && (d->dtype == QL_F32 || d->dtype == QL_BF16) &&
           (int)d->act >= QL_ACT_NONE && (int)d->act <= QL_ACT_SILU && d->ldx >= d->k && d->ldw >= d->k;
}

// (the kernels' counters run past a size by up to a few thousand)
bool sizes_fit(const qhead_linear_desc *d) {
    constexpr int most = 0x7fffffff - 65536;
    return d->m <= most && d->k <= most && d->n <= most;
}

// HIP takes fewer than 2^32 threads a launch, and 65535 rows of blocks: launch(first, blocks) over
// `size` elements, `each` a block, at most `most` blocks a launch.
template <typename F> void in_launches(int size, int each, long long most, const F &launch) {
    for (long long first = 0; first < size; first += most * each)
        launch((int)first, (unsigned)std::min<long long>(most, cdiv(size - first, each)));
}

// --- one product ------------------------------------------------------------------------
// An operand as the caller has it: `rows` rows of `cols` elements.  NAT: t is the row index.
struct Operand {
    const void *p;
    long long rows, cols, ld;
    bool padded;  // (one of our own copies: whole vectors, zeros behind each row)
};

int vec(ql_dtype t) { return t == QL_BF16 ? 8 : 4; }
long long padded_cols(const Operand &o, ql_dtype t) { return (o.cols + vec(t) - 1) / vec(t) * vec(t); }

// Rows of whole 16-byte vectors, whose offsets within a tile fit a buffer resource.
bool direct(const Operand &o, ql_dtype t, bool ptr_aligned) {
    return (o.padded || (o.cols % vec(t) == 0 && o.ld % vec(t) == 0 && ptr_aligned)) &&
           (double)o.ld * (double)esize(t) * 256 < 2147483648.0;
}
bool pad_fits(const Operand &o, ql_dtype t) { return (double)padded_cols(o, t) * (double)esize(t) * 256 < 2147483648.0; }

struct Product {
    int I, J, R;
    Operand a, b;
};

enum Tile { TILE_ANY, TILE_FEW, TILE_64, TILE_128, TILE_256 };
int tile_rows(Tile t) { return t == TILE_256 ? 256 : 128; }
int tile_cols(Tile t) { return t == TILE_256 ? 256 : t == TILE_128 ? 128 : 64; }
int tile_threads(Tile t) { return t == TILE_256 ? 512 : 256; }
struct ProductPlan {
    Tile tile;
    bool pad_a, pad_b;
    int ti, tj, splits, per;
    size_t a_bytes, b_bytes, part_bytes;
    size_t bytes() const { return a_bytes + b_bytes + part_bytes; }
};

// Time of a product in us by tile and splits: rounds of the workgroups over the CUs, each with its ramp and
// epilogue; per K step of 64 bytes, also where two share a CU, kStepUs; the partial sums go out and come
// back at 4.5 TB/s, and joining them is a launch.  Fitted on 30 shapes from 64 x 4096 x 4096 to 8192 x 8192 x 8192.
// 256 x 256 tiles copy the fewest bytes per product; the small ones are for outputs of few tiles
// (1021 x 1537, 1000 deep, fp32: 200 tiles of 128 x 64 fill the CUs without a split).
constexpr double kStepUs[2][3] = {{0.54, 1.03, 3.66}, {0.20, 0.30, 0.86}};  // fp32, bf16; tiles 64, 128, 256
double product_cost(const Product &q, ql_dtype t, Tile tile, int splits) {
    const int steps = cdiv(q.R, 64 / (int)esize(t));
    const double wgs = (double)cdiv(q.I, tile_rows(tile)) * cdiv(q.J, tile_cols(tile)) * splits;
    const double join = splits > 1 ? 3.5 + 8.0 * splits * (double)q.I * q.J / 4.5e6 : 0.0;
    return (tile == TILE_256 ? 8.0 : 5.0) + kStepUs[t == QL_BF16][tile - TILE_64] * cdiv(steps, splits) * std::ceil(wgs / kNumCUs) + join;
}
// ... of the kernel for any layout, which loads element by element (64 x 64 tiles, four workgroups a CU)
double any_cost(const Product &q, ql_dtype t) {
    return 4.0 + 1.6 * cdiv(q.R, 64 / (int)esize(t)) * std::ceil((double)cdiv(q.I, 64) * cdiv(q.J, 64) / (4 * kNumCUs));
}

// al_a, al_b: whether the operands' pointers are (taken to be) 16-byte aligned.  km: both operands have t
// contiguous.
ProductPlan plan_product(const Product &q, ql_dtype t, bool km, bool al_a, bool al_b) {
    ProductPlan p{};
    p.splits = 1;
    const int forced = env_override("QHEAD_TILE", 0);
    // Up to 16 rows the weights are read in place, whatever their layout (1 row of 4096, 4096 outputs, bf16:
    // 11 us a call from Python; 128 x 128 tiles over 8 splits 13).
    if (km && q.I <= 16 && !forced) {
        p.tile = TILE_FEW;
        return p;
    }
    p.pad_a = !direct(q.a, t, al_a);
    p.pad_b = !direct(q.b, t, al_b);
    const bool fits = (!p.pad_a || pad_fits(q.a, t)) && (!p.pad_b || pad_fits(q.b, t));
    if (!fits || q.R == 0 || forced == 1) {
        p.pad_a = p.pad_b = false;
        return p;
    }
    const int steps = cdiv(q.R, 64 / (int)esize(t));
    const double cap = (double)kMaxSplitBytes / (4.0 * q.I * q.J);
    double best = 1e30;
    int want = 1;
    for (Tile tile : {TILE_64, TILE_128, TILE_256})
        for (int s = 1; s == 1 || (s <= 16 && 4 * s <= steps && s <= cap); ++s) {
            const double c = product_cost(q, t, tile, s);
            // (a launch takes fewer than 2^32 threads; 256 x 256 tiles of any output that fits the memory do)
            const double threads = (double)cdiv(q.I, tile_rows(tile)) * cdiv(q.J, tile_cols(tile)) * s * tile_threads(tile);
            if (c >= best || threads >= 4294967296.0) continue;
            best = c;
            p.tile = tile;
            want = s;
        }
    // (a copy is a launch of 3 us and more)
    if ((p.pad_a || p.pad_b) && !forced && any_cost(q, t) < best + 3.0 * ((int)p.pad_a + (int)p.pad_b)) {
        p.tile = TILE_ANY;
        p.pad_a = p.pad_b = false;
        return p;
    }
    if (forced) p.tile = forced == 256 ? TILE_256 : forced == 128 ? TILE_128 : TILE_64;
    want = std::min(std::max(1, env_override("QHEAD_SPLITS", want)), steps);
    p.ti = cdiv(q.I, tile_rows(p.tile));
    p.tj = cdiv(q.J, tile_cols(p.tile));
    p.per = cdiv(steps, want);
    p.splits = cdiv(steps, p.per);
    if (p.pad_a) p.a_bytes = align_up((size_t)q.a.rows * padded_cols(q.a, t) * esize(t));
    if (p.pad_b) p.b_bytes = align_up((size_t)q.b.rows * padded_cols(q.b, t) * esize(t));
    if (p.splits > 1) p.part_bytes = align_up((size_t)p.splits * q.I * q.J * sizeof(float));
    return p;
}

// A zero-padded copy of an operand at `to`; o becomes the copy.
template <typename T> ql_status pad_operand(Operand &o, void *to, ql_dtype t, hipStream_t st) {
    const long long cols = padded_cols(o, t);
    hipLaunchKernelGGL((qhead_pad_kernel<T>), dim3(grid_1d(o.rows * cols / vec(t))), dim3(kThreads), 0, st,
                       static_cast<const T *>(o.p), o.ld, o.rows, (int)o.cols, (int)cols, static_cast<T *>(to));
    o.p = to;
    o.ld = cols;
    o.padded = true;
    return hip_status();
}

template <typename T, bool ANAT, bool BNAT>
ql_status launch_product(const ProductPlan &p, const HeadTileArgs &a, hipStream_t st) {
    const HeadGemmArgs &g = a.g;
    if (p.tile == TILE_ANY) {
        in_launches(g.I, 64, (1ll << 31) / kThreads, [&](int i0, unsigned x) {
            in_launches(g.J, 64, 32768, [&](int j0, unsigned y) {
                HeadGemmArgs some = g;
                some.i0 = i0;
                some.j0 = j0;
                hipLaunchKernelGGL((qhead_gemm_any_kernel<T, ANAT, BNAT>), dim3(x, y), dim3(kThreads), 0, st, some);
            });
        });
        return hip_status();
    }
    if (p.tile == TILE_FEW) {
        if constexpr (!ANAT && !BNAT)
            in_launches(g.J, 16, (1ll << 31) / 512, [&](int j0, unsigned x) {
                HeadGemmArgs some = g;
                some.j0 = j0;
                hipLaunchKernelGGL((qhead_few_kernel<T>), dim3(x), dim3(512), 0, st, some);
            });
        return hip_status();
    }
    const dim3 grid((unsigned)(a.ti * a.tj * a.splits));
    if (p.tile == TILE_256)
        hipLaunchKernelGGL((qhead_gemm_kernel<T, ANAT, BNAT, 256, 256, 2, 4, 4, 1, 2>), grid, dim3(512), 0, st, a);
    else if (p.tile == TILE_128)
        hipLaunchKernelGGL((qhead_gemm_kernel<T, ANAT, BNAT, 128, 128, 2, 2, 4, 2, 4>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((qhead_gemm_kernel<T, ANAT, BNAT, 128, 64, 2, 2, 4, 2, 3>), grid, dim3(256), 0, st, a);
    if (a.splits > 1)
        hipLaunchKernelGGL((qhead_join_kernel<T>), dim3(grid_1d((long long)g.I * cdiv(g.J, 8))), dim3(kThreads), 0, st, a);
    return hip_status();
}

template <bool ANAT, bool BNAT>
ql_status run_product(Product q, const HeadOut &o, ql_dtype t, char *ws, size_t ws_bytes, hipStream_t st) {
    if (q.I == 0 || q.J == 0) return QL_OK;
    ProductPlan p = plan_product(q, t, !ANAT && !BNAT, aligned16(q.a.p), aligned16(q.b.p));
    if (p.bytes() > ws_bytes) {
        // (a misaligned pointer that the descriptor does not announce)
        p = ProductPlan{};
        p.splits = 1;
    }
    ql_status s = QL_OK;
    if (p.pad_a) s = t == QL_BF16 ? pad_operand<uint16_t>(q.a, ws, t, st) : pad_operand<float>(q.a, ws, t, st);
    if (s == QL_OK && p.pad_b)
        s = t == QL_BF16 ? pad_operand<uint16_t>(q.b, ws + p.a_bytes, t, st) : pad_operand<float>(q.b, ws + p.a_bytes, t, st);
    if (s != QL_OK) return s;
    const HeadTileArgs a{HeadGemmArgs{q.a.p, q.b.p, q.a.ld, q.b.ld, q.I, q.J, q.R, o, 0, 0}, p.ti, p.tj, p.splits, p.per,
                         reinterpret_cast<float *>(ws + p.a_bytes + p.b_bytes)};
    return t == QL_BF16 ? launch_product<uint16_t, ANAT, BNAT>(p, a, st) : launch_product<float, ANAT, BNAT>(p, a, st);
}

Product fwd_product(const qhead_linear_desc *d, const void *x, const void *w) {
    return {d->m, d->n, d->k, {x, d->m, d->k, d->ldx, false}, {w, d->n, d->k, d->ldw, false}};
}
Product dx_product(const qhead_linear_desc *d, const Operand &dz, const void *w) {
    return {d->m, d->k, d->n, dz, {w, d->n, d->k, d->ldw, false}};
}
Product dw_product(const qhead_linear_desc *d, const Operand &dz, const void *x) {
    return {d->n, d->k, d->m, dz, {x, d->m, d->k, d->ldx, false}};
}

// --- the pass over dy and z ----------------------------------------------------------------
// dz is stored where there is an activation, and as a copy of dy where the products would copy it
// both; rows of whole vectors.
struct DzPlan {
    bool store;
    long long ld;
    int rpp, parts;
    size_t dz_bytes, part_bytes;
};
DzPlan plan_dz(const qhead_linear_desc *d, bool al) {
    DzPlan p;
    const Operand dy{nullptr, d->m, d->n, d->ldy, false};
    p.store = d->act != QL_ACT_NONE || !direct(dy, d->dtype, al);
    p.ld = padded_cols(dy, d->dtype);
    // (up to 64 rows are one part, whose sums are db itself: a launch less)
    p.rpp = d->m <= 64 ? std::max(1, d->m) : std::max(32, cdiv(d->m, 128));
    p.parts = std::max(1, cdiv(d->m, p.rpp));
    p.dz_bytes = p.store ? align_up((size_t)d->m * p.ld * esize(d->dtype)) : 0;
    p.part_bytes = p.parts > 1 ? align_up((size_t)p.parts * d->n * sizeof(float)) : 0;
    return p;
}

template <typename T>
void launch_dz(const qhead_linear_desc *d, const DzPlan &p, const void *dy, const void *z, void *dz, float *part,
               hipStream_t st) {
    hipLaunchKernelGGL((qhead_dz_kernel<T>), dim3(cdiv(d->n, 256), p.parts), dim3(kThreads), 0, st,
                       static_cast<const T *>(dy), d->ldy, static_cast<const T *>(z), (int)d->act, d->m, d->n, p.rpp,
                       static_cast<T *>(dz), p.ld, part);
}

Operand dz_operand(const qhead_linear_desc *d, const DzPlan &p, const void *dy, void *dz) {
    if (p.store) return {dz, d->m, d->n, p.ld, true};
    return {dy, d->m, d->n, d->ldy, false};
}

}  // namespace

extern "C" {

size_t qhead_linear_fwd_workspace_size(const qhead_linear_desc *d) {
    if (!linear_ok(d) || !sizes_fit(d) || d->m == 0) return 0;
    return plan_product(fwd_product(d, nullptr, nullptr), d->dtype, true, !d->unaligned, !d->unaligned).bytes();
}

ql_status qhead_linear_fwd(const qhead_linear_desc *d, const void *x, const void *w, const float *b, const void *r,
                           void *y, void *z, void *workspace, size_t workspace_bytes, void *stream) {
    if (!linear_ok(d) || d->ldy < d->n || (r && d->ldr < d->n)) return QL_EINVAL;
    if (!sizes_fit(d)) return QL_EUNSUPPORTED;
    if (d->m == 0) return QL_OK;
    if (!x || !w || !y) return QL_EINVAL;
    const void *ptrs[] = {x, w, r, y, z};
    for (const void *p : ptrs)
        if (!aligned(p, esize(d->dtype))) return QL_EINVAL;
    if (!aligned(b, 4)) return QL_EINVAL;
    const size_t need = qhead_linear_fwd_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    return run_product<false, false>(fwd_product(d, x, w), HeadOut{y, d->ldy, b, r, d->ldr, z, (int)d->act, false}, d->dtype,
                                     static_cast<char *>(workspace), workspace_bytes, static_cast<hipStream_t>(stream));
}

size_t qhead_linear_bwd_workspace_size(const qhead_linear_desc *d) {
    if (!linear_ok(d) || !sizes_fit(d) || d->ldy < d->n) return 0;
    const bool al = !d->unaligned;
    const DzPlan p = plan_dz(d, al);
    const Operand dz = dz_operand(d, p, nullptr, nullptr);
    // the two products run one after the other on the same piece
    return p.dz_bytes + p.part_bytes + std::max(plan_product(dx_product(d, dz, nullptr), d->dtype, false, al, al).bytes(),
                                                plan_product(dw_product(d, dz, nullptr), d->dtype, false, al, al).bytes());
}

ql_status qhead_linear_bwd(const qhead_linear_desc *d, const void *x, const void *w, const void *dy, const void *z,
                           void *dx, void *dw, float *db, void *workspace, size_t workspace_bytes, void *stream) {
    if (!linear_ok(d) || d->ldy < d->n) return QL_EINVAL;
    if (d->m > 0 && !dx && !dw && !db) return QL_EINVAL;  // (of no rows dx is no pointer)
    if (!sizes_fit(d)) return QL_EUNSUPPORTED;
    if (d->m == 0 && !dw && !db) return QL_OK;
    if (d->m > 0 && (!dy || (d->act != QL_ACT_NONE && !z) || (dx && !w) || (dw && !x))) return QL_EINVAL;
    const void *ptrs[] = {x, w, dy, z, dx};
    for (const void *p : ptrs)
        if (!aligned(p, esize(d->dtype))) return QL_EINVAL;
    if (!aligned(dw, d->dw_f32 ? 4 : esize(d->dtype)) || !aligned(db, 4)) return QL_EINVAL;
    const size_t need = qhead_linear_bwd_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const DzPlan p = plan_dz(d, !d->unaligned);
    char *ws = static_cast<char *>(workspace);
    void *dz = p.store && (dx || dw) ? ws : nullptr;
    float *part = db && p.parts > 1 ? reinterpret_cast<float *>(ws + p.dz_bytes) : db;
    if (dz || db) {
        if (d->dtype == QL_BF16) launch_dz<uint16_t>(d, p, dy, z, dz, part, st);
        else launch_dz<float>(d, p, dy, z, dz, part, st);
        if (db && p.parts > 1)
            in_launches(d->n, 32, (1ll << 31) / kThreads, [&](int j0, unsigned x) {
                hipLaunchKernelGGL(qhead_colsum_kernel<>, dim3(x), dim3(kThreads), 0, st, part, p.parts, d->n, j0, db);
            });
        const ql_status s = hip_status();
        if (s != QL_OK) return s;
    }
    const Operand src = dz_operand(d, p, dy, dz);
    ws += p.dz_bytes + p.part_bytes;
    const size_t left = workspace_bytes - p.dz_bytes - p.part_bytes;
    if (dx) {
        const ql_status s = run_product<false, true>(dx_product(d, src, w), HeadOut{dx, d->k, nullptr, nullptr, 0, nullptr, QL_ACT_NONE, false},
                                                     d->dtype, ws, left, st);
        if (s != QL_OK) return s;
    }
    if (dw)
        return run_product<true, true>(dw_product(d, src, x), HeadOut{dw, d->k, nullptr, nullptr, 0, nullptr, QL_ACT_NONE, d->dw_f32 != 0},
                                       d->dtype, ws, left, st);
    return QL_OK;
}

}  // extern "C"
