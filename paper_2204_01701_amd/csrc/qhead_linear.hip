// qhead_linear.hip -- host side of the first-order layer of include/qhead.h.
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

template <bool ANAT, bool BNAT> ql_status run_gemm(const HeadGemmArgs &g, ql_dtype dt, hipStream_t st) {
    if (g.I == 0 || g.J == 0) return QL_OK;
    const dim3 grid(cdiv(g.J, 64), cdiv(g.I, 64));
    if (grid.y > 65535) return QL_EUNSUPPORTED;
    if (dt == QL_BF16)
        hipLaunchKernelGGL((qhead_gemm_any_kernel<uint16_t, ANAT, BNAT>), grid, dim3(kThreads), 0, st, g);
    else
        hipLaunchKernelGGL((qhead_gemm_any_kernel<float, ANAT, BNAT>), grid, dim3(kThreads), 0, st, g);
    return hip_status();
}

// The pass over dy and z: rows of a part, parts, and the workspace's pieces.
struct DzPlan {
    bool store;
    int rpp, parts;
    size_t dz_bytes, part_bytes;
};
DzPlan plan_dz(const qhead_linear_desc *d) {
    DzPlan p;
    p.store = d->act != QL_ACT_NONE;
    p.rpp = std::max(32, cdiv(d->m, 256));
    p.parts = std::max(1, cdiv(d->m, p.rpp));
    p.dz_bytes = p.store ? align_up((size_t)d->m * d->n * esize(d->dtype)) : 0;
    p.part_bytes = align_up((size_t)p.parts * d->n * sizeof(float));
    return p;
}

template <typename T>
void launch_dz(const qhead_linear_desc *d, const DzPlan &p, const void *dy, const void *z, void *dz, float *part,
               hipStream_t st) {
    hipLaunchKernelGGL((qhead_dz_kernel<T>), dim3(cdiv(d->n, 64), p.parts), dim3(kThreads), 0, st,
                       static_cast<const T *>(dy), d->ldy, static_cast<const T *>(z), (int)d->act, d->m, d->n, p.rpp,
                       static_cast<T *>(dz), part);
}

}  // namespace

extern "C" {

size_t qhead_linear_fwd_workspace_size(const qhead_linear_desc *d) {
    (void)d;
    return 0;
}

ql_status qhead_linear_fwd(const qhead_linear_desc *d, const void *x, const void *w, const float *b, const void *r,
                           void *y, void *z, void *workspace, size_t workspace_bytes, void *stream) {
    if (!linear_ok(d) || d->ldy < d->n || (r && d->ldr < d->n)) return QL_EINVAL;
    if (d->m == 0) return QL_OK;
    if (!x || !w || !y) return QL_EINVAL;
    const void *ptrs[] = {x, w, r, y, z};
    for (const void *p : ptrs)
        if (!aligned(p, esize(d->dtype))) return QL_EINVAL;
    if (!aligned(b, 4)) return QL_EINVAL;
    const size_t need = qhead_linear_fwd_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    HeadGemmArgs g{x, w, d->ldx, d->ldw, d->m, d->n, d->k, HeadOut{y, d->ldy, b, r, d->ldr, z, (int)d->act}};
    return run_gemm<false, false>(g, d->dtype, static_cast<hipStream_t>(stream));
}

size_t qhead_linear_bwd_workspace_size(const qhead_linear_desc *d) {
    if (!linear_ok(d) || d->ldy < d->n) return 0;
    const DzPlan p = plan_dz(d);
    return p.dz_bytes + p.part_bytes;
}

ql_status qhead_linear_bwd(const qhead_linear_desc *d, const void *x, const void *w, const void *dy, const void *z,
                           void *dx, void *dw, float *db, void *workspace, size_t workspace_bytes, void *stream) {
    if (!linear_ok(d) || d->ldy < d->n) return QL_EINVAL;
    if (!dx && !dw && !db) return QL_EINVAL;
    if (d->m > 0 && (!dy || (d->act != QL_ACT_NONE && !z) || (dx && !w) || (dw && !x))) return QL_EINVAL;
    const void *ptrs[] = {x, w, dy, z, dx, dw};
    for (const void *p : ptrs)
        if (!aligned(p, esize(d->dtype))) return QL_EINVAL;
    if (!aligned(db, 4)) return QL_EINVAL;
    const size_t need = qhead_linear_bwd_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const DzPlan p = plan_dz(d);
    char *ws = static_cast<char *>(workspace);
    void *dz = p.store && (dx || dw) ? ws : nullptr;
    float *part = db ? reinterpret_cast<float *>(ws + p.dz_bytes) : nullptr;
    if (dz || part) {
        if (d->dtype == QL_BF16) launch_dz<uint16_t>(d, p, dy, z, dz, part, st);
        else launch_dz<float>(d, p, dy, z, dz, part, st);
        if (db) hipLaunchKernelGGL(qhead_colsum_kernel<>, dim3(cdiv(d->n, kThreads)), dim3(kThreads), 0, st, part, p.parts, d->n, db);
        const ql_status s = hip_status();
        if (s != QL_OK) return s;
    }
    const void *src = p.store ? dz : dy;
    const long long ld = p.store ? d->n : d->ldy;
    if (dx) {
        HeadGemmArgs g{src, w, ld, d->ldw, d->m, d->k, d->n, HeadOut{dx, d->k, nullptr, nullptr, 0, nullptr, QL_ACT_NONE}};
        const ql_status s = run_gemm<false, true>(g, d->dtype, st);
        if (s != QL_OK) return s;
    }
    if (dw) {
        HeadGemmArgs g{src, x, ld, d->ldx, d->n, d->k, d->m, HeadOut{dw, d->k, nullptr, nullptr, 0, nullptr, QL_ACT_NONE}};
        return run_gemm<true, true>(g, d->dtype, st);
    }
    return QL_OK;
}

}  // extern "C"
