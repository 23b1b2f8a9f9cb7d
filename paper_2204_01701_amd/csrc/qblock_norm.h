// qblock_norm.h -- group normalization with an activation over channels-last maps
// (include/qblock.h), forward and backward.
//
// A pixel's channels are contiguous, a group's values are cpg neighbours of each of hw pixels.  A
// workgroup takes a segment of whole groups (or a part of a very wide one) of one or more samples.
// Its threads form a grid: thread = (sample, pixel lane, column of eight channels), columns and
// lanes powers of two, so a thread keeps its channels while it walks over pixels, a wave reads whole lines, and sums
// over pixels are exchanges between lanes before they are anything else.
//
// Bound by memory.  Where a sample's segment fits the registers of a workgroup it is read once:
// statistics in two passes over registers (mean, then squares of differences to it), then the
// output.  Elsewhere the pixels are cut into chunks: one launch leaves each chunk's statistics,
// another joins them and reads the map again, of which the memory-side cache holds up to 256 MB.
#pragma once

#include "qblock_keep.h"

namespace ql {

struct NormArgs {
    const void *x, *dy;
    void *out;  // y or dx
    const float *gamma, *beta;
    float *mean, *rstd;  // forward: written; backward: read
    int8_t *q;           // forward: written; backward: read in x's place
    uint8_t *e;
    float2 *part;  // [sample][slice][group]: (mean, sum of squares about it), or the sums of t and t xh
    float2 *chan;  // [slot * chunks + chunk][c]: sums of dz and dz xh
    int n, hw, c, groups, cpg;
    int gps, parts, part_c, segs;  // groups of a segment; parts of a group, their channels; segments
    int svl, pnl;                  // log2 of columns, of pixel lanes of a sample
    int chunks, chunk_px, slots;   // slots: workgroups that share the samples
    int blocks, act;
    float eps;
};

// What is the same for a whole workgroup: its segment, its pixels.
struct NormSeg {
    int slot, chunk, part, g0, ng, c0, cn, wide;  // wide: channels of a group within the segment
    int p0, p1;
    __device__ __forceinline__ explicit NormSeg(const NormArgs &a) {
        // (neighbouring segments share cache lines: one XCD takes them)
        int b = xcd_remap(blockIdx.x, a.blocks);
        const int seg = b % a.segs;
        b /= a.segs;
        chunk = b % a.chunks;
        slot = b / a.chunks;
        part = 0;
        if (a.parts == 1) {
            g0 = seg * a.gps;
            ng = min(a.gps, a.groups - g0);
            c0 = g0 * a.cpg;
            cn = ng * a.cpg;
            wide = a.cpg;
        } else {
            g0 = seg / a.parts;
            part = seg - g0 * a.parts;
            ng = 1;
            c0 = g0 * a.cpg + part * a.part_c;
            cn = min(a.part_c, a.cpg - part * a.part_c);
            wide = cn;
        }
        p0 = chunk * a.chunk_px;
        p1 = (int)min((long long)a.hw, (long long)p0 + a.chunk_px);
    }
};

// Eight neighbours as they lie in memory (n of them; zeros behind).
template <typename T> struct NormRaw {
    v4u w[8 / Elem<T>::VEC];
    __device__ __forceinline__ void load(const T *p, int n) {
        if (n >= 8) {
#pragma unroll
            for (int h = 0; h < 8 / Elem<T>::VEC; ++h) w[h] = *reinterpret_cast<const v4u_row *>(p + h * Elem<T>::VEC);
        } else {
            float f[8];
            head_load8<T>(p, f, n);
#pragma unroll
            for (int h = 0; h < 8 / Elem<T>::VEC; ++h) w[h] = vpack<T>(f + h * Elem<T>::VEC);
        }
    }
    __device__ __forceinline__ float get(int i) const { return vget<T>(w[i / Elem<T>::VEC], i % Elem<T>::VEC); }
};

// Thread's place.  U: channels that surely share a group (8 where cpg is a multiple of 8, else 1).
template <int U, int TH> struct NormThread {
    static constexpr int F = 8 / U;  // groups' shares a thread tells apart
    int v, p, sn, col, n8, snl;
    int gi[F];
    __device__ __forceinline__ NormThread(const NormArgs &a, const NormSeg &s) {
        const int tid = threadIdx.x, pl = tid >> a.svl;
        v = tid & ((1 << a.svl) - 1);
        p = pl & ((1 << a.pnl) - 1);
        sn = pl >> a.pnl;
        snl = __builtin_ctz(TH) - a.svl - a.pnl;
        col = 8 * v;
        n8 = s.cn - col;
#pragma unroll
        for (int f = 0; f < F; ++f) gi[f] = min((col + f * U) / s.wide, s.ng - 1);
    }
};

// Sums over each group of each sample: val[k] are this thread's shares, on return sum[k * TH * F + sample * ng + group].
// red and sum hold NV * TH * F floats each.
template <int NV, int U, int TH>
__device__ __forceinline__ void norm_group_sums(const NormArgs &a, const NormSeg &s, const NormThread<U, TH> &t, float (&val)[NV][8 / U],
                                                float *red, float *sum) {
    constexpr int F = 8 / U;
    const int top = min(6, a.svl + a.pnl), pin = max(top - a.svl, 0);
    for (int b = a.svl; b < top; ++b)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int f = 0; f < F; ++f) val[k][f] += __shfl_xor(val[k][f], 1 << b);
    const int rows = 1 << (a.pnl - pin), cols = 1 << a.svl;
    if ((t.p & ((1 << pin) - 1)) == 0) {
        const int at = ((t.sn * rows + (t.p >> pin)) * cols + t.v) * F;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int f = 0; f < F; ++f) red[k * TH * F + at + f] = val[k][f];
    }
    __syncthreads();
    const int items = s.ng << t.snl, each = s.wide / U;
    int lanes = 64;
    while (lanes > 1 && items * lanes > TH) lanes >>= 1;
    const int l = threadIdx.x & (lanes - 1);
    for (int it = threadIdx.x / lanes; it < items; it += TH / lanes) {
        const int sn = it / s.ng, g = it - sn * s.ng;
        float u[NV] = {};
        for (int r = 0; r < rows; ++r) {
            const float *p = red + (sn * rows + r) * cols * F + g * each;
            for (int i = l; i < each; i += lanes)
#pragma unroll
                for (int k = 0; k < NV; ++k) u[k] += p[k * TH * F + i];
        }
        for (int b = 1; b < lanes; b <<= 1)
#pragma unroll
            for (int k = 0; k < NV; ++k) u[k] += __shfl_xor(u[k], b);
        if (l == 0)
#pragma unroll
            for (int k = 0; k < NV; ++k) sum[k * TH * F + it] = u[k];
    }
    __syncthreads();
}

__device__ __forceinline__ void norm_channels(const float *p, int c, int n8, float other, float *v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p && i < n8 ? p[c + i] : other;
}

// y of eight neighbours: stored, and their x into the checkpoint where there is one (every lane of a
// quad comes here; n = 0: nothing to store).
template <typename T>
__device__ __forceinline__ void norm_put(const NormArgs &a, long long pixel, int c, int n, float *x, const float *y) {
    if (n > 0) head_store8<T>(static_cast<T *>(a.out) + pixel * a.c + c, y, n);
    if (!a.q) return;
    if (n < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? x[i] : 0.0f;
    }
    uint32_t e;
    const v2u b = keep_pack8(x, e);
    if (n <= 0) return;
    keep_put8(a.q + pixel * a.c + c, b, n);
    if (c % kKeep == 0) a.e[pixel * ((a.c + kKeep - 1) / kKeep) + c / kKeep] = (uint8_t)e;
}

// Forward.  FUSED: a sample's segment in registers (R pixels a thread), read once.  Else the statistics of a
// chunk: those of its first R pixels a thread in two passes; the rest adds sums of differences, and of their
// squares, to the first mean (which, with at least 1/f of the chunk behind it, costs at most f roundings of the variance).
template <typename T, int R, int U, bool FUSED, int TH>
__global__ __launch_bounds__(TH) void qblock_norm_fwd_kernel(NormArgs a) {
    constexpr int F = 8 / U;
    __shared__ float red[2 * TH * F], sum[2 * TH * F];
    const NormSeg s(a);
    const NormThread<U, TH> t(a, s);
    float gam[8], bet[8];
    if constexpr (FUSED) {
        norm_channels(a.gamma, s.c0 + t.col, t.n8, 1.0f, gam);
        norm_channels(a.beta, s.c0 + t.col, t.n8, 0.0f, bet);
    }
    for (long long ng = s.slot; (ng << t.snl) < a.n; ng += a.slots) {
        const long long sample = (ng << t.snl) + t.sn, pixel0 = sample * a.hw;
        const T *x = static_cast<const T *>(a.x) + s.c0 + t.col;
        const int last = sample < a.n && t.n8 > 0 ? s.p1 : 0;  // (pixels from `last` on are none of this thread's)
        NormRaw<T> raw[R];
        int px = s.p0 + t.p;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int at = px + (r << a.pnl);
            if (at < last) raw[r].load(x + (pixel0 + at) * a.c, t.n8);
            else raw[r] = NormRaw<T>{};
        }
        float one[1][F] = {};
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) one[0][i / U] += raw[r].get(i);
        norm_group_sums<1, U, TH>(a, s, t, one, red, sum);
        const int first = min(R << a.pnl, s.p1 - s.p0);
        const float count = (float)first * s.wide;
        float mean[F];
#pragma unroll
        for (int f = 0; f < F; ++f) mean[f] = sum[t.sn * s.ng + t.gi[f]] / count;
        if constexpr (FUSED) {
#pragma unroll
            for (int f = 0; f < F; ++f) one[0][f] = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (px + (r << a.pnl) < last)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float d = raw[r].get(i) - mean[i / U];
                        one[0][i / U] += d * d;
                    }
            norm_group_sums<1, U, TH>(a, s, t, one, red, sum);
            float rstd[F];
#pragma unroll
            for (int f = 0; f < F; ++f) rstd[f] = 1.0f / sqrtf(sum[t.sn * s.ng + t.gi[f]] / count + a.eps);
            if (t.p == 0 && last > 0)
#pragma unroll
                for (int f = 0; f < F; ++f)
                    if (f * U < t.n8 && (t.col + f * U) % s.wide == 0) {
                        const long long at = sample * a.groups + s.g0 + t.gi[f];
                        if (a.mean) a.mean[at] = mean[f];
                        if (a.rstd) a.rstd[at] = rstd[f];
                    }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int at = px + (r << a.pnl);
                if (at >= last && !(a.q && at < s.p1)) continue;  // (a checkpoint's quads stay together)
                float v[8], z[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] = raw[r].get(i);
                    z[i] = (v[i] - mean[i / U]) * rstd[i / U] * gam[i] + bet[i];
                }
                head_acts<8>(a.act, z);
                norm_put<T>(a, pixel0 + at, s.c0 + t.col, at < last ? t.n8 : 0, v, z);
            }
        } else {
            float two[2][F] = {};
            // about the first mean: sums of differences behind the first pixels, and of all squares
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (px + (r << a.pnl) < last)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float d = raw[r].get(i) - mean[i / U];
                        two[1][i / U] += d * d;
                    }
            for (px += R << a.pnl; px < s.p1; px += R << a.pnl) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int at = px + (r << a.pnl);
                    if (at < last) raw[r].load(x + (pixel0 + at) * a.c, t.n8);
                }
                float d1[F] = {}, d2[F] = {};  // (sums of sums: their roundings do not add up over a long chunk)
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (px + (r << a.pnl) < last)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float d = raw[r].get(i) - mean[i / U];
                            d1[i / U] += d;
                            d2[i / U] += d * d;
                        }
#pragma unroll
                for (int f = 0; f < F; ++f) two[0][f] += d1[f], two[1][f] += d2[f];
            }
            norm_group_sums<2, U, TH>(a, s, t, two, red, sum);
            if (t.p == 0 && last > 0) {
                const float all = (float)(s.p1 - s.p0) * s.wide;
#pragma unroll
                for (int f = 0; f < F; ++f)
                    if (f * U < t.n8 && (t.col + f * U) % s.wide == 0) {
                        const float d = sum[t.sn * s.ng + t.gi[f]], dd = sum[TH * F + t.sn * s.ng + t.gi[f]], by = d / all;
                        a.part[(sample * (a.chunks * a.parts) + s.chunk * a.parts + s.part) * a.groups + s.g0 + t.gi[f]] =
                            make_float2(mean[f] + by, fmaxf(dd - d * by, 0.0f));
                    }
            }
        }
    }
}

// The chunks' statistics of the segment's groups joined: mean and rstd into LDS, a wave a group.
__device__ __forceinline__ void norm_join_stats(const NormArgs &a, const NormSeg &s, long long sample, float *mean, float *rstd) {
    const int lane = threadIdx.x & 63, slices = a.chunks * a.parts;
    const float total = (float)a.hw * a.cpg;
    for (int g = wave_id(); g < s.ng; g += kThreads / 64) {
        const float2 *p = a.part + sample * slices * a.groups + s.g0 + g;
        float m = 0.0f, q = 0.0f;
        auto count = [&](int i) {
            const int ch = i / a.parts, pt = i - ch * a.parts;
            return (float)min(a.chunk_px, a.hw - ch * a.chunk_px) * (a.parts == 1 ? a.cpg : min(a.part_c, a.cpg - pt * a.part_c));
        };
        for (int i = lane; i < slices; i += 64) m += count(i) * p[(size_t)i * a.groups].x;
        for (int b = 1; b < 64; b <<= 1) m += __shfl_xor(m, b);
        m /= total;
        for (int i = lane; i < slices; i += 64) {
            const float2 x = p[(size_t)i * a.groups];
            const float d = x.x - m;
            q += x.y + count(i) * d * d;
        }
        for (int b = 1; b < 64; b <<= 1) q += __shfl_xor(q, b);
        if (lane == 0) {
            mean[g] = m;
            rstd[g] = 1.0f / sqrtf(q / total + a.eps);
        }
    }
    __syncthreads();
}

constexpr int kNormGroups = 2048;  // groups of a segment, at most (its channels)

// The second launch of the forward in chunks.
template <typename T, int U> __global__ __launch_bounds__(kThreads) void qblock_norm_apply_kernel(NormArgs a) {
    __shared__ float lm[kNormGroups], lr[kNormGroups];
    const NormSeg s(a);
    const NormThread<U, kThreads> t(a, s);
    float gam[8], bet[8];
    norm_channels(a.gamma, s.c0 + t.col, t.n8, 1.0f, gam);
    norm_channels(a.beta, s.c0 + t.col, t.n8, 0.0f, bet);
    for (long long sample = s.slot; sample < a.n; sample += a.slots) {
        __syncthreads();
        norm_join_stats(a, s, sample, lm, lr);
        if (s.chunk == 0 && s.part == 0)
            for (int g = threadIdx.x; g < s.ng; g += kThreads) {
                if (a.mean) a.mean[sample * a.groups + s.g0 + g] = lm[g];
                if (a.rstd) a.rstd[sample * a.groups + s.g0 + g] = lr[g];
            }
        float mean[8 / U], rstd[8 / U];
#pragma unroll
        for (int f = 0; f < 8 / U; ++f) mean[f] = lm[t.gi[f]], rstd[f] = lr[t.gi[f]];
        const T *x = static_cast<const T *>(a.x) + s.c0 + t.col;
        for (int px = s.p0 + t.p; px < s.p1; px += 4 << a.pnl) {
            NormRaw<T> raw[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = px + (r << a.pnl);
                if (at < s.p1 && t.n8 > 0) raw[r].load(x + (sample * a.hw + at) * a.c, t.n8);
                else raw[r] = NormRaw<T>{};
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = px + (r << a.pnl);
                if (at >= s.p1) continue;
                float v[8], z[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] = raw[r].get(i);
                    z[i] = (v[i] - mean[i / U]) * rstd[i / U] * gam[i] + bet[i];
                }
                head_acts<8>(a.act, z);
                norm_put<T>(a, sample * a.hw + at, s.c0 + t.col, t.n8, v, z);
            }
        }
    }
}

// --- backward ------------------------------------------------------------------------------
// Eight neighbours of dy and of x, or of its checkpoint.
template <typename T, bool KEPT> struct NormPair {
    NormRaw<T> dy, x;
    __device__ __forceinline__ void load(const NormArgs &a, long long pixel, int c, int n) {
        dy.load(static_cast<const T *>(a.dy) + pixel * a.c + c, n);
        x.load(static_cast<const T *>(a.x) + pixel * a.c + c, n);
    }
    __device__ __forceinline__ void values(float *g, float *v) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = dy.get(i), v[i] = x.get(i);
    }
};
template <typename T> struct NormPair<T, true> {
    NormRaw<T> dy;
    v2u q;
    uint32_t e;
    __device__ __forceinline__ void load(const NormArgs &a, long long pixel, int c, int n) {
        dy.load(static_cast<const T *>(a.dy) + pixel * a.c + c, n);
        // (a segment may begin inside a block, and the eight values then lie in two: see below)
        q = keep_get8(a.q + pixel * a.c + c, n);
        const uint8_t *p = a.e + pixel * ((a.c + kKeep - 1) / kKeep) + c / kKeep;
        e = p[0];
        if (c % 8 && c % kKeep > kKeep - 8 && n > kKeep - c % kKeep) e |= (uint32_t)p[1] << 8;
        else e |= e << 8;
        e |= (uint32_t)(c % kKeep) << 16;
    }
    __device__ __forceinline__ void values(float *g, float *v) const {
        const float s0 = keep_scale(e & 255u), s1 = keep_scale((e >> 8) & 255u);
        const int here = kKeep - (int)(e >> 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            g[i] = dy.get(i);
            v[i] = (float)(int8_t)(q[i >> 2] >> (8 * (i & 3))) * (i < here ? s0 : s1);
        }
    }
};

// dz and xh of eight neighbours.
template <int U, int F>
__device__ __forceinline__ void norm_slopes(int act, const float (&mean)[F], const float (&rstd)[F], const float *gam, const float *bet,
                                            float *g, float *x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (x[i] - mean[i / U]) * rstd[i / U];
    if (act != HEAD_NONE) {
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = x[i] * gam[i] + bet[i];
        head_slopes<8>(act, z, g);
    }
}

// Backward.  FUSED: a sample's segment of dy and x in registers, read once, and dx.  Else the sums of a chunk.
// Either way the channels' sums over the workgroup's samples and pixels go to a.chan.
template <typename T, int R, int U, bool FUSED, bool KEPT, int TH>
__global__ __launch_bounds__(TH) void qblock_norm_bwd_kernel(NormArgs a) {
    constexpr int F = 8 / U;
    __shared__ float red[2 * TH * 8], sum[2 * TH * F];
    const NormSeg s(a);
    const NormThread<U, TH> t(a, s);
    const int c = s.c0 + t.col;
    float gam[8], bet[8], c1[8] = {}, c2[8] = {};
    norm_channels(a.gamma, c, t.n8, 1.0f, gam);
    norm_channels(a.beta, c, t.n8, 0.0f, bet);
    for (long long ng = s.slot; (ng << t.snl) < a.n; ng += a.slots) {
        const long long sample = (ng << t.snl) + t.sn, pixel0 = sample * a.hw;
        const int last = sample < a.n && t.n8 > 0 ? s.p1 : 0;
        float mean[F], rstd[F];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const long long at = sample * a.groups + s.g0 + t.gi[f];
            mean[f] = last ? a.mean[at] : 0.0f;
            rstd[f] = last ? a.rstd[at] : 0.0f;
        }
        NormPair<T, KEPT> raw[R];
        float s1[8] = {}, s2[8] = {};
        for (int px = s.p0 + t.p; px < s.p1; px += R << a.pnl) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int at = px + (r << a.pnl);
                if (at < last) raw[r].load(a, pixel0 + at, c, t.n8);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (px + (r << a.pnl) >= last) continue;
                float g[8], x[8];
                raw[r].values(g, x);
                norm_slopes<U, F>(a.act, mean, rstd, gam, bet, g, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) s1[i] += g[i], s2[i] += g[i] * x[i];
            }
            if constexpr (FUSED) break;  // (R pixels a thread are all there are)
        }
        float two[2][F] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c1[i] += s1[i], c2[i] += s2[i];
            two[0][i / U] += gam[i] * s1[i];
            two[1][i / U] += gam[i] * s2[i];
        }
        if (!a.out) continue;
        norm_group_sums<2, U, TH>(a, s, t, two, red, sum);
        if constexpr (FUSED) {
            const float inv = 1.0f / ((float)a.hw * a.cpg);
            float ta[F], tx[F];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                ta[f] = sum[t.sn * s.ng + t.gi[f]] * inv;
                tx[f] = sum[TH * F + t.sn * s.ng + t.gi[f]] * inv;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int at = s.p0 + t.p + (r << a.pnl);
                if (at >= last) continue;
                float g[8], x[8];
                raw[r].values(g, x);
                norm_slopes<U, F>(a.act, mean, rstd, gam, bet, g, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = rstd[i / U] * (gam[i] * g[i] - ta[i / U] - x[i] * tx[i / U]);
                head_store8<T>(static_cast<T *>(a.out) + (pixel0 + at) * a.c + c, g, t.n8);
            }
        } else if (t.p == 0 && last > 0) {
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (f * U < t.n8 && (t.col + f * U) % s.wide == 0)
                    a.part[(sample * (a.chunks * a.parts) + s.chunk * a.parts + s.part) * a.groups + s.g0 + t.gi[f]] =
                        make_float2(sum[t.sn * s.ng + t.gi[f]], sum[TH * F + t.sn * s.ng + t.gi[f]]);
        }
    }
    if (!a.chan) return;
    // the channels' sums over the lanes of every sample and pixel
    for (int b = a.svl; b < 6; ++b)
#pragma unroll
        for (int i = 0; i < 8; ++i) c1[i] += __shfl_xor(c1[i], 1 << b), c2[i] += __shfl_xor(c2[i], 1 << b);
    const int pin = max(6 - a.svl, 0), pl = threadIdx.x >> a.svl, wide = 8 << a.svl, rows = TH >> (a.svl + pin);
    __syncthreads();
    if ((pl & ((1 << pin) - 1)) == 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            red[(pl >> pin) * wide + t.col + i] = c1[i];
            red[TH * 8 + (pl >> pin) * wide + t.col + i] = c2[i];
        }
    __syncthreads();
    for (int j = threadIdx.x; j < s.cn; j += TH) {
        float u = 0.0f, w = 0.0f;
        for (int r = 0; r < rows; ++r) u += red[r * wide + j], w += red[TH * 8 + r * wide + j];
        a.chan[((size_t)s.slot * a.chunks + s.chunk) * a.c + s.c0 + j] = make_float2(u, w);
    }
}

// The second launch of the backward in chunks.
template <typename T, int U, bool KEPT> __global__ __launch_bounds__(kThreads) void qblock_norm_dx_kernel(NormArgs a) {
    constexpr int F = 8 / U;
    __shared__ float la[kNormGroups], lx[kNormGroups];
    const NormSeg s(a);
    const NormThread<U, kThreads> t(a, s);
    const int c = s.c0 + t.col, lane = threadIdx.x & 63, slices = a.chunks * a.parts;
    const float inv = 1.0f / ((float)a.hw * a.cpg);
    float gam[8], bet[8];
    norm_channels(a.gamma, c, t.n8, 1.0f, gam);
    norm_channels(a.beta, c, t.n8, 0.0f, bet);
    for (long long sample = s.slot; sample < a.n; sample += a.slots) {
        __syncthreads();
        for (int g = wave_id(); g < s.ng; g += kThreads / 64) {
            const float2 *p = a.part + sample * slices * a.groups + s.g0 + g;
            float u = 0.0f, w = 0.0f;
            for (int i = lane; i < slices; i += 64) {
                const float2 x = p[(size_t)i * a.groups];
                u += x.x, w += x.y;
            }
            for (int b = 1; b < 64; b <<= 1) u += __shfl_xor(u, b), w += __shfl_xor(w, b);
            if (lane == 0) la[g] = u * inv, lx[g] = w * inv;
        }
        __syncthreads();
        float mean[F], rstd[F], ta[F], tx[F];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const long long at = sample * a.groups + s.g0 + t.gi[f];
            mean[f] = a.mean[at];
            rstd[f] = a.rstd[at];
            ta[f] = la[t.gi[f]];
            tx[f] = lx[t.gi[f]];
        }
        if (t.n8 <= 0) continue;
        for (int px = s.p0 + t.p; px < s.p1; px += 2 << a.pnl) {
            NormPair<T, KEPT> raw[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int at = px + (r << a.pnl);
                if (at < s.p1) raw[r].load(a, sample * a.hw + at, c, t.n8);
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int at = px + (r << a.pnl);
                if (at >= s.p1) continue;
                float g[8], x[8];
                raw[r].values(g, x);
                norm_slopes<U, F>(a.act, mean, rstd, gam, bet, g, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = rstd[i / U] * (gam[i] * g[i] - ta[i / U] - x[i] * tx[i / U]);
                head_store8<T>(static_cast<T *>(a.out) + (sample * a.hw + at) * a.c + c, g, t.n8);
            }
        }
    }
}

// dgamma and dbeta from `rows` partial sums a channel: 32 channels a workgroup, 32 rows at a time, four requested
// together.
template <int = 0>
__global__ __launch_bounds__(1024) void qblock_norm_param_kernel(const float2 *chan, int rows, int c, float *dgamma, float *dbeta) {
    __shared__ float2 sum[32][33];
    const int j = blockIdx.x * 32 + (threadIdx.x & 31), r0 = threadIdx.x >> 5;
    float u = 0.0f, w = 0.0f;
    if (j < c)
        for (int r = r0; r < rows; r += 128) {
            float2 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = r + 32 * k < rows ? chan[(size_t)(r + 32 * k) * c + j] : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < 4; ++k) u += x[k].x, w += x[k].y;
        }
    sum[r0][threadIdx.x & 31] = make_float2(u, w);
    __syncthreads();
    // column k of the sums is joined by half a wave
    const int k = threadIdx.x >> 5;
    float2 x = sum[threadIdx.x & 31][k];
    for (int b = 1; b < 32; b <<= 1) x.x += __shfl_xor(x.x, b), x.y += __shfl_xor(x.y, b);
    const int to = blockIdx.x * 32 + k;
    if ((threadIdx.x & 31) || to >= c) return;
    if (dbeta) dbeta[to] = x.x;
    if (dgamma) dgamma[to] = x.y;
}

}  // namespace ql
