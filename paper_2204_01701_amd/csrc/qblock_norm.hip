// qblock_norm.hip -- host side of the group normalization of include/qblock.h.
#include <cmath>

#include "qblock_norm_host.h"

using namespace ql;
using namespace ql::host;

namespace {

bool norm_ok(const qblock_norm_desc *d) {
    return d && d->n >= 0 && d->hw > 0 && d->c > 0 && d->groups > 0 && d->c % d->groups == 0 && float_type(d->dtype) && known_act(d->act);
}
bool sizes_fit(const qblock_norm_desc *d) {
    return d->n <= kMostInt && d->hw <= kMostInt && d->c <= 1 << 20 && (double)d->n * d->hw * d->c < 140737488355328.0;
}

// The samples over workgroups: SN of them at once, `most` workgroups a segment and chunk at most, but a multiple of these where each
// would take more than `run` batches (a multiple, for equal shares on the CUs: 2^18 x 16 x 256 in 1306 us, 1571 with as few as it takes).
void share_samples(NormPlan &p, int n, long long most, long long run) {
    // Outputs are streamed where a workgroup writes whole rows, or at least 64 bytes (bf16) or 128 (float32) of one:
    // 128 x 1024 x 256, bf16, forward 45 to 35 us; 512 x 49 x 512, float32, 28 to 22.  Lesser parts of lines lose by it: 32
    // bytes in bf16 77 to 94 us, 64 in float32 62 to 74.
    const int line = p.a.gps * p.a.cpg * p.es;
    p.a.stream = p.a.segs == 1 || p.a.parts > 1 || line >= (p.es == 2 ? 64 : 128);
    const int snl = log2_up(p.th) - p.a.svl - p.a.pnl;
    const long long groups = ((long long)n + (1LL << snl) - 1) >> snl;
    const long long times = std::max(1LL, (groups + run * most - 1) / (run * most));
    p.a.slots = (int)std::max(1LL, std::min(groups, most * times));
    p.a.blocks = (int)((long long)p.a.slots * p.a.chunks * p.a.segs);
    p.a.by_segs = make_fastdiv(p.a.segs);
    p.a.by_chunks = make_fastdiv(p.a.chunks);
    p.a.by_wide = make_fastdiv(p.a.cpg);
}

// Batches of samples whose channels' sums the backward adds up one by one, in registers' form and in chunks (whose own sums are up to
// 128 terms long).  2^20 rows of 4096 took 2048 of them, whose roundings cost up to 492 x 2^-24 of a sum; a.chan then has 8 bytes a
// channel more for each of these runs, at most a fiftieth of x.
constexpr long long kRunFused = 192, kRunChunks = 64, kNoRun = 1LL << 32;

// bwd: the backward's plan (its registers hold dy as well, its workgroups share few lines of a.chan).
NormPlan plan_norm(const qblock_norm_desc *d, bool bwd) {
    NormPlan p{};
    NormArgs &a = p.a;
    const int cpg = d->c / d->groups, es = (int)esize(d->dtype);
    a.n = d->n, a.hw = d->hw, a.c = d->c, a.groups = d->groups, a.cpg = cpg;
    a.act = (int)d->act, a.eps = d->eps;
    p.u = cpg % 8 == 0 ? 8 : cpg % 4 == 0 ? 4 : cpg % 2 == 0 ? 2 : 1;
    p.es = es;
    a.parts = 1, a.part_c = cpg;
    auto segment = [&](int gps) {
        a.gps = std::max(1, std::min(d->groups, gps));
        a.segs = cdiv(d->groups, a.gps);
        a.svl = log2_up(((long long)a.gps * cpg + 7) / 8);
    };
    // Registers.  Time of a candidate in us: a launch, then the values of a workgroup at `each` ns (fitted on 12 maps from
    // 1 x 1024 x 512 to 128 x 1024 x 256 and 8192 rows of 1024; segments of a line of 128, 64 or 32 bytes, of which the XCD's L2
    // joins neighbours), in rounds over the CUs; that of chunks with their further launches likewise.  It ranks the candidates of one
    // map and is no prediction: a value costs the same in either type, so that it says 51 for the forward of 128 x 1024 x 256, which
    // takes 33 in bf16 and 69 in float32.
    const double values = (double)std::max(1, d->n) * d->hw * d->c, each = 1e-3 * (bwd ? (p.u == 8 ? 0.45 : 1.2) : (p.u == 8 ? 0.35 : 0.7));
    double best = (bwd ? 13.0 : 10.0) + 1.3 * each * values / kNumCUs;
    const int forced = env_override("QBLOCK_NORM_FUSED", -1), forced_line = env_override("QBLOCK_NORM_LINE", 0);
    if (forced == 1) best = 1e300;
    const int most_r = !bwd && d->dtype == QL_F32 ? 16 : 8;
    int line_at = 0, th_at = 0;
    if (cpg <= 8 * 512 && forced != 0)
        for (int line : {128, 64, 32}) {
            if (forced_line && line != forced_line) continue;
            segment(cdiv(line, cpg * es));
            for (int th : {256, 512}) {
                const int lth = log2_up(th);
                if (a.svl > lth) continue;
                const long long need = (d->hw + (1LL << (lth - a.svl)) - 1) >> (lth - a.svl);
                if (need > (th == 256 ? 8 : most_r) || (need > 8 && line < 64)) continue;
                const double wgs = std::max(1.0, (double)std::max(1, d->n) * a.segs), rounds = wgs / kNumCUs;
                // (a float's line of 32 bytes is a single column: 134 us where 128 bytes take 125)
                const double form = es == 4 && line == 32 ? 2.2 : 1.0;
                const double t = 5.0 + form * each * values / wgs * (rounds < 4 ? std::ceil(rounds) : rounds);
                if (t < 0.97 * best) best = t, line_at = line, th_at = th;
                break;
            }
        }
    if (line_at) {
        segment(cdiv(line_at, cpg * es));
        const int lth = log2_up(th_at);
        const long long need = (d->hw + (1LL << (lth - a.svl)) - 1) >> (lth - a.svl);
        a.pnl = lth - a.svl;
        p.r = need <= 2 ? 2 : need <= 8 ? 8 : 16;
        // several samples a workgroup, as long as their lanes have room
        while (a.pnl > 0 && ((long long)p.r << (a.pnl - 1)) >= d->hw) --a.pnl;
        if ((double)(1 << (lth - a.svl - a.pnl)) * d->hw * d->c * es < 2147483648.0) {  // (a thread's offset)
            p.fused = true;
            p.th = th_at;
            a.chunks = 1;
            a.chunk_px = d->hw;
            share_samples(p, d->n, bwd ? std::max(1, cdiv(4 * kNumCUs, a.segs)) : (1 << 20) / a.segs + 1, bwd ? kRunFused : kNoRun);
            if (bwd) p.chan_bytes = align_up((size_t)a.slots * d->c * sizeof(float2));
            return p;
        }
    }
    // Chunks: segments of up to 512 channels, or a part of a group of up to 2048.
    p.th = kThreads;
    if (cpg > 2048) {
        a.gps = 1;
        a.part_c = 2048;
        a.parts = cdiv(cpg, 2048);
        a.segs = d->groups * a.parts;
        a.svl = 8;
    } else {
        segment(512 / cpg);
    }
    a.pnl = 8 - a.svl;
    // steps of the workgroup's pixel lanes: at most 128 a chunk (a thread's sums stay short), else what gives every CU four workgroups
    const long long steps = (d->hw + (1LL << a.pnl) - 1) >> a.pnl, all = steps * std::max(1, d->n) * a.segs;
    // (two where the map is small or the groups' channels are told apart: 24 us for 2 x 50176 x 64 in 32 groups, 31 with four)
    const int wgs = env_override("QBLOCK_NORM_WGS", p.u == 8 && values >= 8e6 ? 4 * kNumCUs : 2 * kNumCUs);
    const long long per = std::max(1LL, std::min(128LL, (all + wgs - 1) / wgs));
    p.r = per <= 2 ? 2 : 8;
    a.chunk_px = (int)std::min<long long>(d->hw, per << a.pnl);
    a.chunks = cdiv(d->hw, a.chunk_px);
    share_samples(p, d->n, bwd ? std::max(1LL, 8LL * kNumCUs / ((long long)a.segs * a.chunks)) : (1LL << 22) / ((long long)a.segs * a.chunks) + 1,
                  bwd ? kRunChunks : kNoRun);
    p.part_bytes = align_up((size_t)std::max(1, d->n) * a.chunks * a.parts * d->groups * sizeof(float2));
    p.joined_bytes = align_up((size_t)std::max(1, d->n) * d->groups * sizeof(float2));  // (mean and rstd, or the two averages)
    if (bwd) p.chan_bytes = align_up((size_t)a.slots * a.chunks * d->c * sizeof(float2));
    return p;
}

// Whether the forward's launches can write the checkpoint on the way: segments of whole blocks, whose lanes are quads.  (Else
// a launch of its own does: the plan, and with it the order of the sums, is the same with a checkpoint and without.)
bool emits(const NormPlan &p) { return p.a.parts == 1 && (p.a.segs == 1 || p.a.gps * p.a.cpg % kKeep == 0) && p.a.svl >= 2; }

template <int = 0> __global__ __launch_bounds__(kThreads) void qblock_zero_kernel(float *p, float *q, int n) {
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < n; i += gridDim.x * kThreads) {
        if (p) p[i] = 0.0f;
        if (q) q[i] = 0.0f;
    }
}

}  // namespace

extern "C" {

size_t qblock_norm_fwd_workspace_size(const qblock_norm_desc *d) {
    if (!norm_ok(d) || !sizes_fit(d) || d->n == 0) return 0;
    return plan_norm(d, false).bytes();
}

ql_status qblock_norm_fwd(const qblock_norm_desc *d, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                          float *rstd, int8_t *q, uint8_t *e, void *workspace, size_t workspace_bytes, void *stream) {
    if (!norm_ok(d) || !(d->eps > 0.0f) || !std::isfinite(d->eps)) return QL_EINVAL;
    if (!sizes_fit(d)) return QL_EUNSUPPORTED;
    if (d->n == 0) return QL_OK;
    if (!x || !y || !q != !e) return QL_EINVAL;
    if (!aligned(x, esize(d->dtype)) || !aligned(y, esize(d->dtype))) return QL_EINVAL;
    const void *floats[] = {gamma, beta, mean, rstd};
    for (const void *p : floats)
        if (!aligned(p, 4)) return QL_EINVAL;
    const size_t need = qblock_norm_fwd_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const NormPlan p = plan_norm(d, false);
    NormArgs a = p.a;
    a.x = x, a.out = y, a.gamma = gamma, a.beta = beta, a.mean = mean, a.rstd = rstd;
    a.part = static_cast<float2 *>(workspace);
    float *stats = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.part_bytes);
    if (!p.fused && !a.mean) a.mean = stats;
    if (!p.fused && !a.rstd) a.rstd = stats + (size_t)d->n * d->groups;
    if (q && emits(p)) {
        a.q = q, a.e = e;
    } else if (q) {  // (first: y may be x)
        const ql_status s = run_keep(true, d->dtype, const_cast<void *>(x), d->c, q, e, (long long)d->n * d->hw, d->c, st);
        if (s != QL_OK) return s;
    }
    return launch_norm_fwd(d->dtype, p, a, st);
}

size_t qblock_norm_bwd_workspace_size(const qblock_norm_desc *d) {
    if (!norm_ok(d) || !sizes_fit(d) || d->n == 0) return 0;
    return plan_norm(d, true).bytes();
}

ql_status qblock_norm_bwd(const qblock_norm_desc *d, const void *dy, const void *x, const int8_t *q, const uint8_t *e, const float *gamma,
                          const float *beta, const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *workspace,
                          size_t workspace_bytes, void *stream) {
    if (!norm_ok(d)) return QL_EINVAL;
    if (d->n > 0 && !dx && !dgamma && !dbeta) return QL_EINVAL;  // (of an empty map dx is no pointer)
    if (!sizes_fit(d)) return QL_EUNSUPPORTED;
    const size_t es = esize(d->dtype);
    if (d->n > 0 && (!dy || (!x && (!q || !e)) || !mean || !rstd)) return QL_EINVAL;
    if (!aligned(dy, es) || !aligned(x, es) || !aligned(dx, es)) return QL_EINVAL;
    const void *floats[] = {gamma, beta, mean, rstd, dgamma, dbeta};
    for (const void *p : floats)
        if (!aligned(p, 4)) return QL_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d->n == 0) {
        if (!dgamma && !dbeta) return QL_OK;
        hipLaunchKernelGGL(qblock_zero_kernel<>, dim3(grid_1d(d->c)), dim3(kThreads), 0, st, dgamma, dbeta, d->c);
        return hip_status();
    }
    const size_t need = qblock_norm_bwd_workspace_size(d);
    if (workspace_bytes < need || (need && !workspace)) return QL_EWORKSPACE;
    if (workspace && !aligned16(workspace)) return QL_EINVAL;
    const NormPlan p = plan_norm(d, true);
    NormArgs a = p.a;
    a.x = x, a.dy = dy, a.out = dx, a.gamma = gamma, a.beta = beta;
    a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd);
    a.part = static_cast<float2 *>(workspace);
    a.avg = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + p.part_bytes);
    if (dgamma || dbeta) a.chan = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + p.part_bytes + p.joined_bytes);
    const bool kept = x == nullptr;
    if (kept) a.q = const_cast<int8_t *>(q), a.e = const_cast<uint8_t *>(e);
    if (d->dtype == QL_BF16) launch_norm_bwd_of<uint16_t>(p, a, kept, st);
    else launch_norm_bwd_of<float>(p, a, kept, st);
    if (a.chan)
        hipLaunchKernelGGL(qblock_norm_param_kernel<>, dim3(cdiv(a.c, 16)), dim3(1024), 0, st, a.chan, a.slots * a.chunks, a.c, dgamma, dbeta);
    return hip_status();
}

}  // extern "C"
