// qhead_rows.hip -- host side of the rows-of-logits operators of include/qhead.h:
// argument checks, the split of few long rows over workgroups, launches.
#include <cmath>

#include "qhead.h"
#include "qhead_rows.h"
#include "qhost.h"

using namespace ql;
using namespace ql::host;

namespace {

constexpr int kRowThreads = 256;

// Rows enough to fill the GPU with one wave each (eight a CU at least).
bool many_rows(int rows) { return rows >= 8 * kNumCUs; }

// (log2(e) / T is a factor of every exponent: infinite, it would make the largest logit's 0 a NaN)
bool rows_ok(const qhead_rows_desc *d) {
    return d && d->rows >= 0 && d->vocab > 0 && d->ld >= d->vocab && (d->dtype == QL_F32 || d->dtype == QL_BF16) &&
           std::isfinite(d->temperature) && d->temperature > 0.0f && std::isfinite(kLog2e / d->temperature);
}
bool top_ok(const qhead_rows_desc *d) { return d->top >= 0 && d->top <= QHEAD_MAX_TOP && d->top <= d->vocab; }
// (T^2 is a factor of the loss)
bool places_ok(const qhead_rows_desc *d) {
    return d->top >= 0 && d->top <= QHEAD_MAX_TOP && d->alpha >= 0.0f && d->alpha <= 1.0f &&
           std::isfinite(d->temperature * d->temperature);
}
size_t esize(ql_dtype t) { return t == QL_BF16 ? 2 : 4; }
int vec(ql_dtype t) { return t == QL_BF16 ? 8 : 4; }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int vectors(const qhead_rows_desc *d) { return (int)(((long long)d->vocab + vec(d->dtype) - 1) / vec(d->dtype)); }

// Few rows: parts of `per` vectors of a row, so that about `blocks` workgroups share the work.
struct Split {
    int splits, per;
};
Split split_rows(int rows, int nvec, int blocks, int most, int least_per) {
    const int want = std::max(1, std::min({cdiv(blocks, rows), most, nvec / least_per}));
    const int per = want == 1 ? nvec : cdiv(cdiv(nvec, want), kRowThreads) * kRowThreads;
    return {cdiv(nvec, per), per};
}

// A part of a row has two vectors a thread at least.  (Parts of the alternatives' lists
// together fit the join's 16 KiB.)
Split logprobs_split(const qhead_rows_desc *d) {
    if (d->rows >= kNumCUs) return {1, vectors(d)};
    const int most = std::min(kHeadMaxSplits, kHeadJoinKeys / std::max(1, d->top));
    return split_rows(d->rows, vectors(d), 2 * kNumCUs, most, 2 * kRowThreads);
}
Split sums_split(const qhead_rows_desc *d) {
    if (d->rows >= kNumCUs) return {1, vectors(d)};
    return split_rows(d->rows, vectors(d), 2 * kNumCUs, kHeadMaxSplits, 2 * kRowThreads);
}
Split grad_split(const qhead_rows_desc *d) { return split_rows(d->rows, vectors(d), 4 * kNumCUs, 1 << 16, 2 * kRowThreads); }

// launch(args, grid) over all rows, `threads` each: HIP takes fewer than 2^32 threads a launch, so
// rows beyond half of that go into further ones (rows so many are not split).
template <typename A, typename F> void over_rows(A a, int rows, int threads, const F &launch) {
    const int most = (int)((1ll << 31) / threads);
    for (; a.row0 < rows; a.row0 += most)
        launch(a, dim3((unsigned)(std::min<long long>(most, rows - a.row0) * a.splits)));
}

template <typename T, int TH, int U, bool TOP> void launch_logprobs_as(const HeadLogprobArgs &all, int rows, hipStream_t st) {
    over_rows(all, rows, TH, [&](const HeadLogprobArgs &a, dim3 grid) {
        hipLaunchKernelGGL((qhead_logprobs_kernel<T, TH, U, TOP>), grid, dim3(TH), 0, st, a);
    });
}
template <typename T> void launch_logprobs(const HeadLogprobArgs &a, int rows, hipStream_t st) {
    const int nvec = cdiv((long long)a.V, Elem<T>::VEC);
    // One wave where a row is at most one vector a lane, or short and one of many, unless K is large for the bound
    // that its few lanes' maxima give (4000 rows of 700, K = 64, bf16: 64 us, four waves 20).
    const bool one = nvec <= 64, wave = nvec <= 1024 && 4 * a.K <= nvec && many_rows(rows);
    if (a.K) {
        if (one) launch_logprobs_as<T, 64, 1, true>(a, rows, st);
        else if (wave) launch_logprobs_as<T, 64, 4, true>(a, rows, st);
        else launch_logprobs_as<T, kRowThreads, 4, true>(a, rows, st);
    } else {
        if (one) launch_logprobs_as<T, 64, 1, false>(a, rows, st);
        else if (wave) launch_logprobs_as<T, 64, 4, false>(a, rows, st);
        else launch_logprobs_as<T, kRowThreads, 4, false>(a, rows, st);
    }
    if (a.splits > 1)
        hipLaunchKernelGGL((qhead_logprobs_join_kernel<T>), dim3(rows), dim3(256), (size_t)a.splits * a.K * 8, st, a);
}

template <typename T> void launch_logprobs_grad(const HeadLogprobGradArgs &all, int rows, hipStream_t st) {
    over_rows(all, rows, kRowThreads, [&](const HeadLogprobGradArgs &a, dim3 grid) {
        if (a.h) hipLaunchKernelGGL((qhead_logprobs_grad_kernel<T, kRowThreads, 4, true>), grid, dim3(kRowThreads), 0, st, a);
        else hipLaunchKernelGGL((qhead_logprobs_grad_kernel<T, kRowThreads, 4, false>), grid, dim3(kRowThreads), 0, st, a);
    });
}

// Which sums a distillation needs: those at T alone, those at T = 1 alone, or both (`two`).
struct Terms {
    bool teacher, label, two;
};
Terms distill_terms(const qhead_rows_desc *d, const int64_t *label) {
    Terms t;
    t.teacher = d->top > 0 && d->alpha > 0.0f;
    t.label = label && d->alpha < 1.0f;
    t.two = t.teacher && t.label && d->temperature != 1.0f;
    return t;
}

ql_status distill_args(const qhead_rows_desc *d, const void *logits, const int64_t *t_ids, const void *t_logits,
                       const int64_t *label, HeadDistillArgs &a) {
    if (!rows_ok(d) || !places_ok(d)) return QL_EINVAL;
    if (d->rows == 0) return QL_OK;
    if (!logits || (d->top && (!t_ids || !t_logits))) return QL_EINVAL;
    if (!aligned(logits, esize(d->dtype)) || !aligned(t_logits, d->teacher_f32 ? 4 : esize(d->dtype)) || !aligned(t_ids, 8) || !aligned(label, 8))
        return QL_EINVAL;
    const Terms t = distill_terms(d, label);
    a.z = logits;
    a.ld = d->ld;
    a.V = d->vocab;
    a.K = t.teacher ? d->top : 0;
    a.temp = d->temperature;
    a.inv_t = 1.0f / d->temperature;
    a.c = t.teacher ? kLog2e / d->temperature : kLog2e;
    a.alpha = d->alpha;
    a.ids = t_ids;
    a.tz = t_logits;
    a.tz_f32 = d->teacher_f32 != 0;
    a.label = t.label ? label : nullptr;
    return QL_OK;
}

template <typename T, int TH, int U, bool TWO, bool GRAD, bool HELD>
void launch_row_as(const HeadDistillArgs &all, int rows, hipStream_t st) {
    over_rows(all, rows, TH, [&](const HeadDistillArgs &a, dim3 grid) {
        hipLaunchKernelGGL((qhead_distill_row_kernel<T, TH, U, TWO, GRAD, HELD>), grid, dim3(TH), 0, st, a);
    });
}
// The kernel of a workgroup per row by the row's length in vectors.  One wave where a row is short and rows
// are many (8192 rows of 1000, bf16, step: 24 us against 57 with 256 threads; 4096 of 8000: 45 and 49).  The
// step holds a row in registers, up to 16 vectors a thread, as far as a workgroup reaches: 4096 rows of 131072,
// bf16, 457 us against 650 (256 threads) and 524 (1024, fewer rows under way, which the caches still hold) read
// twice; 2048 of 32768, fp32, 114 against 145.  Where two sums make it compute-bound (bf16, label and
// teacher at a temperature) 16 vectors on 1024 threads lose to the second read: 559 against 524.  16 vectors on
// fewer threads beat 8 on more (1023 of 50001, bf16, both terms: 68 against 83; 4096 of 32768: 133, 146), but
// not in fp32 up to 4096 vectors (2048 of 16000: 65, 60).
template <typename T, bool TWO, bool GRAD> void launch_row(const HeadDistillArgs &a, int rows, hipStream_t st) {
    const int nvec = cdiv((long long)a.V, Elem<T>::VEC);
    const bool many = many_rows(rows);
    if (nvec <= 64) return launch_row_as<T, 64, 1, TWO, GRAD, GRAD>(a, rows, st);
    if (nvec <= 256 && many) return launch_row_as<T, 64, 4, TWO, GRAD, GRAD>(a, rows, st);
    if (nvec <= 1024) {
        if (many) return launch_row_as<T, 64, 4, TWO, GRAD, false>(a, rows, st);
        return launch_row_as<T, kRowThreads, 4, TWO, GRAD, GRAD>(a, rows, st);
    }
    if constexpr (GRAD) {
        if (nvec <= 2048) return launch_row_as<T, 256, 8, TWO, GRAD, true>(a, rows, st);
        if (nvec <= 4096) {
            if constexpr (sizeof(T) == 2) return launch_row_as<T, 256, 16, TWO, GRAD, true>(a, rows, st);
            else return launch_row_as<T, 512, 8, TWO, GRAD, true>(a, rows, st);
        }
        if (nvec <= 8192) return launch_row_as<T, 512, 16, TWO, GRAD, true>(a, rows, st);
        if constexpr (!(TWO && sizeof(T) == 2))
            if (nvec <= 16384) return launch_row_as<T, 1024, 16, TWO, GRAD, true>(a, rows, st);
        return launch_row_as<T, 1024, 2, TWO, GRAD, false>(a, rows, st);
    }
    launch_row_as<T, kRowThreads, 4, TWO, GRAD, false>(a, rows, st);
}
template <typename T, bool TWO> void launch_parts(const HeadDistillArgs &a, int rows, hipStream_t st) {
    hipLaunchKernelGGL((qhead_distill_part_kernel<T, kRowThreads, 4, TWO>), dim3(rows * a.splits), dim3(kRowThreads), 0, st, a);
    hipLaunchKernelGGL((qhead_distill_join_kernel<T, TWO>), dim3(rows), dim3(64), 0, st, a);
}
template <typename T, bool TWO> void launch_distill_grad(const HeadDistillArgs &all, int rows, hipStream_t st) {
    over_rows(all, rows, kRowThreads, [&](const HeadDistillArgs &a, dim3 grid) {
        hipLaunchKernelGGL((qhead_distill_grad_kernel<T, kRowThreads, 4, TWO>), grid, dim3(kRowThreads), 0, st, a);
    });
}

// FN<T, TWO>(args...) for the descriptor's type
#define HEAD_DISPATCH(FN, two, dt, ...)                                \
    do {                                                               \
        if ((dt) == QL_BF16) {                                         \
            if (two) FN<uint16_t, true>(__VA_ARGS__);                  \
            else FN<uint16_t, false>(__VA_ARGS__);                     \
        } else {                                                       \
            if (two) FN<float, true>(__VA_ARGS__);                     \
            else FN<float, false>(__VA_ARGS__);                        \
        }                                                              \
    } while (0)

template <typename T, bool TWO> void launch_row_loss(const HeadDistillArgs &a, int rows, hipStream_t st) {
    launch_row<T, TWO, false>(a, rows, st);
}
template <typename T, bool TWO> void launch_row_step(const HeadDistillArgs &a, int rows, hipStream_t st) {
    launch_row<T, TWO, true>(a, rows, st);
}

}  // namespace

extern "C" {

size_t qhead_logprobs_fwd_workspace_size(const qhead_rows_desc *d) {
    if (!rows_ok(d) || !top_ok(d) || d->rows == 0) return 0;
    const Split s = logprobs_split(d);
    if (s.splits == 1) return 0;
    const size_t parts = (size_t)d->rows * s.splits;
    return align_up(parts * sizeof(HeadSums)) + align_up(parts * d->top * sizeof(uint64_t));
}

ql_status qhead_logprobs_fwd(const qhead_rows_desc *d, const void *logits, const int64_t *target, float *logp,
                             float *entropy, float *lse, float *top_logp, int64_t *top_ids, float *stats,
                             void *workspace, size_t workspace_bytes, void *stream) {
    if (!rows_ok(d) || !top_ok(d)) return QL_EINVAL;
    if (d->rows == 0) return QL_OK;
    if (!logits || !target || !logp || (d->top && (!top_logp || !top_ids))) return QL_EINVAL;
    const void *p4[] = {logp, entropy, lse, top_logp, stats}, *p8[] = {target, top_ids};
    for (const void *p : p4)
        if (!aligned(p, 4)) return QL_EINVAL;
    for (const void *p : p8)
        if (!aligned(p, 8)) return QL_EINVAL;
    if (!aligned(logits, esize(d->dtype))) return QL_EINVAL;
    const size_t need = qhead_logprobs_fwd_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    const Split s = logprobs_split(d);
    HeadLogprobArgs a{};
    a.z = logits;
    a.ld = d->ld;
    a.V = d->vocab;
    a.K = d->top;
    a.splits = s.splits;
    a.per = s.per;
    a.c = kLog2e / d->temperature;
    a.inv_t = 1.0f / d->temperature;
    a.target = target;
    a.logp = logp;
    a.entropy = entropy;
    a.lse = lse;
    a.top_logp = top_logp;
    a.top_ids = top_ids;
    a.stats = stats;
    if (need) {
        a.part = static_cast<HeadSums *>(workspace);
        a.part_top = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) +
                                                  align_up((size_t)d->rows * s.splits * sizeof(HeadSums)));
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d->dtype == QL_BF16) launch_logprobs<uint16_t>(a, d->rows, st);
    else launch_logprobs<float>(a, d->rows, st);
    return hip_status();
}

ql_status qhead_logprobs_bwd(const qhead_rows_desc *d, const void *logits, const int64_t *target, const float *stats,
                             const float *entropy, const float *g, const float *h, void *dlogits, void *stream) {
    if (!rows_ok(d)) return QL_EINVAL;
    if (d->rows == 0) return QL_OK;
    if (!logits || !target || !stats || !g || !dlogits || (h && !entropy)) return QL_EINVAL;
    if (dlogits == logits && d->ld != d->vocab) return QL_EINVAL;
    const void *p4[] = {stats, entropy, g, h};
    for (const void *p : p4)
        if (!aligned(p, 4)) return QL_EINVAL;
    if (!aligned(target, 8) || !aligned(logits, esize(d->dtype)) || !aligned(dlogits, esize(d->dtype))) return QL_EINVAL;
    const Split s = grad_split(d);
    const HeadLogprobGradArgs a{logits, d->ld, 0, d->vocab, s.splits, s.per, kLog2e / d->temperature, 1.0f / d->temperature,
                                target, stats, entropy, g, h, dlogits};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d->dtype == QL_BF16) launch_logprobs_grad<uint16_t>(a, d->rows, st);
    else launch_logprobs_grad<float>(a, d->rows, st);
    return hip_status();
}

size_t qhead_distill_workspace_size(const qhead_rows_desc *d) {
    if (!rows_ok(d) || !places_ok(d) || d->rows == 0) return 0;
    const Split s = sums_split(d);
    if (s.splits == 1) return 0;
    return align_up((size_t)d->rows * s.splits * sizeof(HeadSums)) + align_up((size_t)d->rows * 4 * sizeof(float));
}

ql_status qhead_distill_fwd(const qhead_rows_desc *d, const void *logits, const int64_t *t_ids, const void *t_logits,
                            const int64_t *label, float *loss, float *stats, void *workspace, size_t workspace_bytes,
                            void *stream) {
    HeadDistillArgs a{};
    const ql_status ok = distill_args(d, logits, t_ids, t_logits, label, a);
    if (ok != QL_OK || d->rows == 0) return ok;
    if (!loss || !aligned(loss, 4) || !aligned(stats, 4)) return QL_EINVAL;
    const size_t need = qhead_distill_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    const Split s = sums_split(d);
    a.splits = s.splits;
    a.per = s.per;
    a.loss = loss;
    a.stats = stats;
    a.part = static_cast<HeadSums *>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool two = distill_terms(d, label).two;
    if (s.splits == 1) HEAD_DISPATCH(launch_row_loss, two, d->dtype, a, d->rows, st);
    else HEAD_DISPATCH(launch_parts, two, d->dtype, a, d->rows, st);
    return hip_status();
}

ql_status qhead_distill_bwd(const qhead_rows_desc *d, const void *logits, const int64_t *t_ids, const void *t_logits,
                            const int64_t *label, const float *stats, const float *g, void *dlogits, void *stream) {
    HeadDistillArgs a{};
    const ql_status ok = distill_args(d, logits, t_ids, t_logits, label, a);
    if (ok != QL_OK || d->rows == 0) return ok;
    if (!stats || !g || !dlogits || (dlogits == logits && d->ld != d->vocab)) return QL_EINVAL;
    if (!aligned(stats, 4) || !aligned(g, 4) || !aligned(dlogits, esize(d->dtype))) return QL_EINVAL;
    const Split s = grad_split(d);
    a.splits = s.splits;
    a.per = s.per;
    a.stats = const_cast<float *>(stats);
    a.g = g;
    a.dz = dlogits;
    hipStream_t st = static_cast<hipStream_t>(stream);
    HEAD_DISPATCH(launch_distill_grad, distill_terms(d, label).two, d->dtype, a, d->rows, st);
    return hip_status();
}

ql_status qhead_distill_step(const qhead_rows_desc *d, const void *logits, const int64_t *t_ids, const void *t_logits,
                             const int64_t *label, const float *g, float *loss, void *dlogits, void *workspace,
                             size_t workspace_bytes, void *stream) {
    HeadDistillArgs a{};
    const ql_status ok = distill_args(d, logits, t_ids, t_logits, label, a);
    if (ok != QL_OK || d->rows == 0) return ok;
    if (!loss || !g || !dlogits || (dlogits == logits && d->ld != d->vocab)) return QL_EINVAL;
    if (!aligned(loss, 4) || !aligned(g, 4) || !aligned(dlogits, esize(d->dtype))) return QL_EINVAL;
    const size_t need = qhead_distill_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    const Split s = sums_split(d);
    a.splits = s.splits;
    a.per = s.per;
    a.loss = loss;
    a.g = g;
    a.dz = dlogits;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool two = distill_terms(d, label).two;
    if (s.splits == 1) {
        HEAD_DISPATCH(launch_row_step, two, d->dtype, a, d->rows, st);
        return hip_status();
    }
    a.part = static_cast<HeadSums *>(workspace);
    a.stats = reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                        align_up((size_t)d->rows * s.splits * sizeof(HeadSums)));
    HEAD_DISPATCH(launch_parts, two, d->dtype, a, d->rows, st);
    const ql_status parts = hip_status();
    if (parts != QL_OK) return parts;
    const Split sg = grad_split(d);
    a.splits = sg.splits;
    a.per = sg.per;
    HEAD_DISPATCH(launch_distill_grad, two, d->dtype, a, d->rows, st);
    return hip_status();
}

}  // extern "C"
