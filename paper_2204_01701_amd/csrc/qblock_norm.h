// qblock_norm.h -- group normalization with an activation over channels-last maps
// (include/qblock.h), forward and backward.
//
// A pixel's channels are contiguous, a group's values are cpg neighbours of each of hw pixels.  A
// workgroup takes a segment of whole groups (or a part of a very wide one) of one or more samples.
// Its threads form a grid: thread = (sample, pixel lane, column of eight channels), columns and
// lanes powers of two, so a thread keeps its channels while it walks over pixels, a wave reads whole lines, and sums
// over pixels are exchanges between lanes before they are anything else.
//
// Large forwards are bound by memory (128 x 1024 x 256 in bf16: 33 us, a copy of its bytes 28).  Backwards in registers are bound by
// neither memory nor the vector ALU: a workgroup of 512 threads has a CU to itself (its values, dz and sums take 222 to 256
// registers), so that its loads, its arithmetic and its stores follow each other.  128 x 1024 x 256 with gelu: bf16 76 us, of which
// a copy of its bytes takes 41 and the vector ALU is busy for 55 %; float32 129, a copy 83, busy for 30 %.  In chunks the slope is
// evaluated in both launches.  Rows of 1024 in bf16 (hw = 1, gelu) keep the vector ALU busy for 89 % of the time forward and
// 77 % backward, at 59 and 52 instructions a value (maps: 34 and 36): half of a thread's two places for pixels stay empty.  Where a sample's segment fits the registers
// of a workgroup it is read once: statistics in two passes over registers (mean, then squares of differences to it), then
// the output.  Elsewhere the pixels are cut into chunks: one launch leaves each chunk's statistics, a small one joins
// them, a third reads the map again, of which the memory-side cache holds up to 256 MB.
#pragma once

#include <type_traits>

#include "qblock_act.h"
#include "qblock_keep.h"

namespace ql {

struct NormArgs {
    const void *x, *dy;
    void *out;  // y or dx
    const float *gamma, *beta;
    float *mean, *rstd;  // forward: written; backward: read
    int8_t *q;           // forward: written; backward: read in x's place
    uint8_t *e;
    float2 *part;  // [sample][slice][group]: (mean, sum of squares about it), or sigma_1 and sigma_2
    float2 *avg;   // [sample][group]: sigma_1 / N and sigma_2 / N
    float2 *chan;  // [slot * chunks + chunk][c]: sums of dz and dz xh
    int n, hw, c, groups, cpg;
    int gps, parts, part_c, segs;  // groups of a segment; parts of a group, their channels; segments
    int svl, pnl;                  // log2 of columns, of pixel lanes of a sample
    int chunks, chunk_px, slots;   // slots: workgroups that share the samples
    int blocks, act;
    bool stream;  // the output's stores are streamed
    float eps;
    FastDiv by_segs, by_chunks, by_wide;  // (wide: channels of a group within a segment, where groups are whole)
};

// What is the same for a whole workgroup: its segment, its pixels.
struct NormSeg {
    int slot, chunk, part, g0, ng, c0, cn, wide;  // wide: channels of a group within the segment
    int p0, p1;
    // Whether eight elements from any channel of the pixels before `end` lie inside the map.
    __device__ __forceinline__ static bool room(const NormArgs &a, long long end) { return end * a.c + 8 <= (long long)a.n * a.hw * a.c; }
    __device__ __forceinline__ explicit NormSeg(const NormArgs &a) {
        // (neighbouring segments share cache lines: one XCD takes them)
        const int b = xcd_remap(blockIdx.x, a.blocks), bs = (int)fdiv((uint32_t)b, a.by_segs), seg = b - bs * a.segs;
        slot = (int)fdiv((uint32_t)bs, a.by_chunks);
        chunk = bs - slot * a.chunks;
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
    // room: eight elements may be read though fewer count (single loads behind branches would wait for each other).
    __device__ __forceinline__ void load(const char *p, int n, bool room) {
        if (n >= 8 || room) {
#pragma unroll
            for (int h = 0; h < 8 / Elem<T>::VEC; ++h) w[h] = *reinterpret_cast<const v4u_row *>(p + h * 16);
        } else {
            float f[8];
            head_load8<T>(reinterpret_cast<const T *>(p), f, n);
#pragma unroll
            for (int h = 0; h < 8 / Elem<T>::VEC; ++h) w[h] = vpack<T>(f + h * Elem<T>::VEC);
        }
    }
    // Zeros behind the n that count (apart from the load: what looks at a value waits for it, and for each load in turn).
    __device__ __forceinline__ void settle(int n) {
        if (n >= 8) return;
        constexpr int D = sizeof(T) == 2 ? 2 : 1;  // elements of a dword
#pragma unroll
        for (int d = 0; d < 8 / D; ++d) {
            const uint32_t x = w[d / 4][d % 4];
            w[d / 4][d % 4] = n >= (d + 1) * D ? x : n <= d * D ? 0u : x & 0xffffu;
        }
    }
    __device__ __forceinline__ float get(int i) const { return vget<T>(w[i / Elem<T>::VEC], i % Elem<T>::VEC); }
    // The bits as they are, and nothing of what was made of them: else the compiler keeps bf16 values converted, in twice the
    // registers, from one pass over them to the next.
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (int h = 0; h < 8 / Elem<T>::VEC; ++h) asm volatile("" : "+v"(w[h]));
    }
};

// Where a thread's pixels lie: an address that is the same for the workgroup, one 32-bit offset of the thread, and a
// step from pixel to pixel that is the workgroup's again, so that a thread needs no addresses of its own.  The host keeps
// the offsets below 2^31 bytes.
struct NormWalk {
    long long at;   // the workgroup's first pixel
    int c, c0;
    int lanes;      // pixels from one step to the next
    uint32_t pix, col;  // the thread's pixel behind the first, its first channel behind c0
    __device__ __forceinline__ NormWalk(const NormArgs &a, int c0_, long long first, uint32_t thread_pixel, int thread_col)
        : at(first), c(a.c), c0(c0_), lanes(1 << a.pnl), pix(thread_pixel), col((uint32_t)thread_col) {}
    template <typename E, typename P> __device__ __forceinline__ P *ptr(P *base, int step) const {
        typedef typename std::conditional<std::is_const<P>::value, const char, char>::type byte;
        byte *b = static_cast<byte *>(base) + ((at + (long long)step * lanes) * c + c0) * (int)sizeof(E);
        return b + (pix * (uint32_t)c + col) * (uint32_t)sizeof(E);
    }
    __device__ __forceinline__ size_t block(int step, int blocks) const {
        return (size_t)(at + (long long)step * lanes + pix) * blocks + (c0 + col) / kKeep;
    }
};

// Thread's place.  U: channels that surely share a group, the largest of 8, 4, 2 and 1 that divides cpg.
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
        for (int f = 0; f < F; ++f) gi[f] = a.parts == 1 ? min((int)fdiv((uint32_t)(col + f * U), a.by_wide), s.ng - 1) : 0;
    }
    // Whether the thread holds its f-th group's first channel.
    __device__ __forceinline__ bool leads(const NormSeg &s, int f) const { return f * U < n8 && col + f * U == gi[f] * s.wide; }
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
    if (p && n8 > 0) {
        head_load8<float>(p + c, v, n8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = other;
    }
}

// y of eight neighbours: stored, and their x into the checkpoint where there is one (every lane of a
// quad comes here; n <= 0: nothing to store).
template <typename T>
__device__ __forceinline__ void norm_put(const NormArgs &a, const NormWalk &w, int step, int n, float *x, const float *y) {
    if (n > 0) block_store8<T>(reinterpret_cast<T *>(w.ptr<T>(static_cast<char *>(a.out), step)), y, n, a.stream);
    if (!a.q) return;
    if (n < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? x[i] : 0.0f;
    }
    uint32_t e;
    const v2u b = keep_pack8(x, e);
    if (n <= 0) return;
    keep_put8(reinterpret_cast<int8_t *>(w.ptr<int8_t>(reinterpret_cast<char *>(a.q), step)), b, n);
    if ((w.c0 + w.col) % kKeep == 0) a.e[w.block(step, (a.c + kKeep - 1) / kKeep)] = (uint8_t)e;
}

// Waves a SIMD that the registers are to leave room for: two workgroups of 512 on a CU where the values held allow it, so that
// one loads while another computes.
template <typename T, int R, int U> constexpr int norm_waves() { return R * (int)sizeof(T) <= 32 && U >= 4 ? 4 : 2; }

// Forward.  FUSED: a sample's segment in registers (R pixels a thread), read once.  Else the statistics of a
// chunk: those of its first R pixels a thread in two passes; the rest adds sums of differences, and of their
// squares, to the first mean (which, with at least 1/f of the chunk behind it, costs at most f roundings of the variance).
template <typename T, int R, int U, bool FUSED, int TH>
__global__ __launch_bounds__(TH, (norm_waves<T, R, U>())) void qblock_norm_fwd_kernel(NormArgs a) {
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
        const long long sample = (ng << t.snl) + t.sn;
        const int last = sample < a.n && t.n8 > 0 ? s.p1 : 0;  // (pixels from `last` on are none of this thread's)
        NormWalk w(a, s.c0, (ng << t.snl) * a.hw + s.p0, (uint32_t)(t.sn * a.hw + t.p), t.col);
        const bool room = NormSeg::room(a, FUSED ? min((ng + 1) << t.snl, (long long)a.n) * a.hw : sample * a.hw + s.p1);
        NormRaw<T> raw[R];
        int px = s.p0 + t.p;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int at = px + (r << a.pnl);
            raw[r] = NormRaw<T>{};
            if (at < last) raw[r].load(w.ptr<T>(static_cast<const char *>(a.x), r), U == 8 ? 8 : t.n8, room);
        }
        if (U < 8)
#pragma unroll
            for (int r = 0; r < R; ++r) raw[r].settle(t.n8);
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
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r].forget();
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
#pragma unroll
            for (int r = 0; r < R; ++r) raw[r].forget();
            float rstd[F];
#pragma unroll
            for (int f = 0; f < F; ++f) rstd[f] = 1.0f / sqrtf(sum[t.sn * s.ng + t.gi[f]] / count + a.eps);
            if (t.p == 0 && last > 0)
#pragma unroll
                for (int f = 0; f < F; ++f)
                    if (t.leads(s, f)) {
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
                block_acts<4>(a.act, z);  // (by fours: fewer registers at a time)
                block_acts<4>(a.act, z + 4);
                norm_put<T>(a, w, r, at < last ? (U == 8 ? 8 : t.n8) : 0, v, z);
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
                w.at += R << a.pnl;
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (px + (r << a.pnl) < last) raw[r].load(w.ptr<T>(static_cast<const char *>(a.x), r), U == 8 ? 8 : t.n8, room);
                if (U < 8)
#pragma unroll
                    for (int r = 0; r < R; ++r) raw[r].settle(t.n8);
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
                    if (t.leads(s, f)) {
                        const float d = sum[t.sn * s.ng + t.gi[f]], dd = sum[TH * F + t.sn * s.ng + t.gi[f]], by = d / all;
                        a.part[(sample * (a.chunks * a.parts) + s.chunk * a.parts + s.part) * a.groups + s.g0 + t.gi[f]] =
                            make_float2(mean[f] + by, fmaxf(dd - d * by, 0.0f));
                    }
            }
        }
    }
}

// Between the two launches over the pixels: the slices of a group of a sample joined, a lane a slice (64 lanes at most), to
// its mean and rstd (STATS), or to the backward's averages.  By itself: in every workgroup of the second launch it
// took up to half of the launch.
template <bool STATS> __global__ __launch_bounds__(kThreads) void qblock_norm_join_kernel(NormArgs a) {
    const int slices = a.chunks * a.parts, lanes = slices > 1 ? 1 << min(6, 32 - __clz(slices - 1)) : 1;
    const int lane = threadIdx.x & (lanes - 1);
    const long long items = (long long)a.n * a.groups, step = (long long)gridDim.x * (kThreads / lanes);
    const float total = (float)a.hw * a.cpg;
    auto count = [&](int i) {
        if (a.parts == 1) return (float)min(a.chunk_px, a.hw - i * a.chunk_px) * a.cpg;
        const int ch = i / a.parts, pt = i - ch * a.parts;
        return (float)min(a.chunk_px, a.hw - ch * a.chunk_px) * min(a.part_c, a.cpg - pt * a.part_c);
    };
    for (long long it = (long long)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes; it < items; it += step) {
        const long long sample = it / a.groups;
        const float2 *p = a.part + sample * slices * a.groups + (it - sample * a.groups);
        float2 x = make_float2(0.0f, 0.0f);  // (a lane's only slice, where there are up to 64)
        float m = 0.0f, q = 0.0f;
        for (int i = lane; i < slices; i += lanes) {
            x = p[(size_t)i * a.groups];
            m += STATS ? count(i) * x.x : x.x;
            if (!STATS) q += x.y;
        }
        for (int b = 1; b < lanes; b <<= 1) m += __shfl_xor(m, b);
        m /= total;
        if constexpr (STATS) {
            for (int i = lane; i < slices; i += lanes) {
                if (slices > lanes) x = p[(size_t)i * a.groups];
                const float d = x.x - m;
                q += x.y + count(i) * d * d;
            }
        }
        for (int b = 1; b < lanes; b <<= 1) q += __shfl_xor(q, b);
        if (lane) continue;
        if constexpr (STATS) {
            a.mean[it] = m;
            a.rstd[it] = 1.0f / sqrtf(q / total + a.eps);
        } else {
            a.avg[it] = make_float2(m, q / total);
        }
    }
}

// The second launch of the forward in chunks.
template <typename T, int U> __global__ __launch_bounds__(kThreads) void qblock_norm_apply_kernel(NormArgs a) {
    const NormSeg s(a);
    const NormThread<U, kThreads> t(a, s);
    float gam[8], bet[8];
    norm_channels(a.gamma, s.c0 + t.col, t.n8, 1.0f, gam);
    norm_channels(a.beta, s.c0 + t.col, t.n8, 0.0f, bet);
    for (long long sample = s.slot; sample < a.n; sample += a.slots) {
        float mean[8 / U], rstd[8 / U];
#pragma unroll
        for (int f = 0; f < 8 / U; ++f) {
            const long long at = sample * a.groups + s.g0 + t.gi[f];
            mean[f] = a.mean[at];
            rstd[f] = a.rstd[at];
        }
        const bool room = NormSeg::room(a, sample * a.hw + s.p1);
        NormWalk w(a, s.c0, sample * a.hw + s.p0, (uint32_t)t.p, t.col);
        for (int px = s.p0 + t.p; px < s.p1; px += 4 << a.pnl, w.at += 4 << a.pnl) {
            NormRaw<T> raw[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                raw[r] = NormRaw<T>{};
                if (px + (r << a.pnl) < s.p1 && t.n8 > 0) raw[r].load(w.ptr<T>(static_cast<const char *>(a.x), r), U == 8 ? 8 : t.n8, room);
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
                block_acts<8>(a.act, z);
                norm_put<T>(a, w, r, t.n8, v, z);
            }
        }
    }
}

// --- backward ------------------------------------------------------------------------------
// Eight neighbours of dy and of x, or of its checkpoint.  U = 8: they lie in one of its blocks; else in up to two.
template <typename T, int U, bool KEPT> struct NormPair {
    NormRaw<T> dy, x;
    __device__ __forceinline__ void load(const NormArgs &a, const NormWalk &w, int step, int n, bool room) {
        dy.load(w.ptr<T>(static_cast<const char *>(a.dy), step), n, room);
        x.load(w.ptr<T>(static_cast<const char *>(a.x), step), n, room);
    }
    __device__ __forceinline__ void settle(int n) {
        if (U == 8) return;
        dy.settle(n);
        x.settle(n);
    }
    __device__ __forceinline__ void gradient(float *g) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = dy.get(i);
    }
    __device__ __forceinline__ void input(const NormWalk &, float *v) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x.get(i);
    }
    __device__ __forceinline__ void forget() { x.forget(); }
};
template <typename T, int U> struct NormPair<T, U, true> {
    NormRaw<T> dy;
    v2u q;
    uint32_t e0, e1;
    __device__ __forceinline__ void load(const NormArgs &a, const NormWalk &w, int step, int n, bool room) {
        dy.load(w.ptr<T>(static_cast<const char *>(a.dy), step), n, room);
        q = keep_get8(reinterpret_cast<const int8_t *>(w.ptr<int8_t>(reinterpret_cast<const char *>(a.q), step)), room ? 8 : n);
        const uint8_t *p = a.e + w.block(step, (a.c + kKeep - 1) / kKeep);
        e0 = p[0];
        if (U < 8) {
            const uint32_t in = (w.c0 + w.col) % kKeep;
            e1 = 0;
            if (in > kKeep - 8 && n > (int)(kKeep - in)) e1 = p[1];
        }
    }
    __device__ __forceinline__ void settle(int n) {  // (q's bytes behind n meet a dy of 0 there)
        if (U < 8) dy.settle(n);
    }
    __device__ __forceinline__ void gradient(float *g) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = dy.get(i);
    }
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(q)); }
    __device__ __forceinline__ void input(const NormWalk &w, float *v) const {
        const float s0 = keep_scale(e0), s1 = U < 8 ? keep_scale(e1) : s0;
        const int here = kKeep - (int)((w.c0 + w.col) % kKeep);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(q[i >> 2] >> (8 * (i & 3))) * (U == 8 || i < here ? s0 : s1);
    }
};

// With d = x - mean and A = gamma rstd: z = A d + beta, and in the sums over a group sigma_1 = sum A dz, sigma_2 = sum A dz d,
//     dx = A dz - sigma_1 / N - d rstd^2 sigma_2 / N,
// which takes three instructions a value less than xh and t do.

// x -> d of eight neighbours; dy -> dz.
template <int U, int F> __device__ __forceinline__ void norm_differences(const float (&mean)[F], float *x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] -= mean[i / U];
}
__device__ __forceinline__ void norm_slopes(int act, const float *scale, const float *bet, const float *d, float *g) {
    if (act != HEAD_NONE) {
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = d[i] * scale[i] + bet[i];
        block_slopes<4>(act, z, g);  // (by fours: fewer registers at a time)
        block_slopes<4>(act, z + 4, g + 4);
    }
}
// Backward.  FUSED: a sample's segment of dy and x in registers, read once, and dx.  Else the sums of a chunk.
// Either way the channels' sums over the workgroup's samples and pixels go to a.chan.
template <typename T, int R, int U, bool FUSED, bool KEPT, int TH>
__global__ __launch_bounds__(TH, FUSED || U < 4 ? 2 : 4) void qblock_norm_bwd_kernel(NormArgs a) {
    constexpr int F = 8 / U;
    __shared__ float red[2 * TH * F], sum[2 * TH * F];
    __shared__ v4f chan[4][TH];  // (each thread's own: its channels' sums over the samples, kept out of its registers)
    const NormSeg s(a);
    const NormThread<U, TH> t(a, s);
    const int c = s.c0 + t.col;
    float bet[8];
#pragma unroll
    for (int h = 0; h < 4; ++h) chan[h][threadIdx.x] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    norm_channels(a.beta, c, t.n8, 0.0f, bet);
    for (long long ng = s.slot; (ng << t.snl) < a.n; ng += a.slots) {
        const long long sample = (ng << t.snl) + t.sn;
        const int last = sample < a.n && t.n8 > 0 ? s.p1 : 0;
        const bool room = NormSeg::room(a, FUSED ? min((ng + 1) << t.snl, (long long)a.n) * a.hw : sample * a.hw + s.p1);
        NormWalk w(a, s.c0, (ng << t.snl) * a.hw + s.p0, (uint32_t)(t.sn * a.hw + t.p), t.col);
        float mean[F], rstd[F];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const long long at = sample * a.groups + s.g0 + t.gi[f];
            mean[f] = last ? a.mean[at] : 0.0f;
            rstd[f] = last ? a.rstd[at] : 0.0f;
        }
        float scale[8];
        norm_channels(a.gamma, c, t.n8, 1.0f, scale);
        auto times_rstd = [&] {  // (behind the loads, which it would wait in front of)
#pragma unroll
            for (int i = 0; i < 8; ++i) scale[i] *= rstd[i / U];
        };
        if (!FUSED) times_rstd();
        NormPair<T, U, KEPT> raw[R];
        float dz[FUSED ? R : 1][8];  // (the slopes cost as much as all else: once, where the values stay)
        float s1[8] = {}, s2[8] = {};
        for (int px = s.p0 + t.p; px < s.p1; px += R << a.pnl, w.at += R << a.pnl) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (px + (r << a.pnl) < last) raw[r].load(a, w, r, U == 8 ? 8 : t.n8, room);
            if (FUSED) times_rstd();
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (px + (r << a.pnl) >= last) continue;
                raw[r].settle(t.n8);
                float *g = dz[FUSED ? r : 0], x[8];
                raw[r].gradient(g);
                raw[r].input(w, x);
                norm_differences<U, F>(mean, x);
                norm_slopes(a.act, scale, bet, x, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) s1[i] += g[i], s2[i] += g[i] * x[i];
                if constexpr (FUSED) raw[r].forget();
            }
            if constexpr (FUSED) break;  // (R pixels a thread are all there are)
        }
        float two[2][F] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            two[0][i / U] += scale[i] * s1[i];
            two[1][i / U] += scale[i] * s2[i];
            s2[i] *= rstd[i / U];
        }
        if (a.chan) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                chan[h][threadIdx.x] += v4f{s1[4 * h], s1[4 * h + 1], s1[4 * h + 2], s1[4 * h + 3]};
                chan[2 + h][threadIdx.x] += v4f{s2[4 * h], s2[4 * h + 1], s2[4 * h + 2], s2[4 * h + 3]};
            }
        }
        if (!a.out) continue;
        norm_group_sums<2, U, TH>(a, s, t, two, red, sum);
        if constexpr (FUSED) {
            const float inv = 1.0f / ((float)a.hw * a.cpg);
            float ta[F], tx[F];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                ta[f] = sum[t.sn * s.ng + t.gi[f]] * inv;
                tx[f] = rstd[f] * (rstd[f] * (sum[TH * F + t.sn * s.ng + t.gi[f]] * inv));
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int at = s.p0 + t.p + (r << a.pnl);
                if (at >= last) continue;
                float *g = dz[r], x[8];
                raw[r].input(w, x);
                norm_differences<U, F>(mean, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = scale[i] * g[i] - (ta[i / U] + x[i] * tx[i / U]);
                block_store8<T>(reinterpret_cast<T *>(w.ptr<T>(static_cast<char *>(a.out), r)), g, U == 8 ? 8 : t.n8, a.stream);
            }
        } else if (t.p == 0 && last > 0) {
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (t.leads(s, f))
                    a.part[(sample * (a.chunks * a.parts) + s.chunk * a.parts + s.part) * a.groups + s.g0 + t.gi[f]] =
                        make_float2(sum[t.sn * s.ng + t.gi[f]], sum[TH * F + t.sn * s.ng + t.gi[f]]);
        }
    }
    if (!a.chan) return;
    // the channels' sums over the lanes of every sample and pixel: first those of a wave, then the waves
    float c1[8], c2[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c1[i] = chan[i >> 2][threadIdx.x][i & 3], c2[i] = chan[2 + (i >> 2)][threadIdx.x][i & 3];
    for (int b = a.svl; b < 6; ++b)
#pragma unroll
        for (int i = 0; i < 8; ++i) c1[i] += __shfl_xor(c1[i], 1 << b), c2[i] += __shfl_xor(c2[i], 1 << b);
    const int pin = max(6 - a.svl, 0), pl = threadIdx.x >> a.svl, wide = 8 << a.svl, rows = TH >> (a.svl + pin);
    float *both = reinterpret_cast<float *>(chan);  // 2 x TH x 8
    __syncthreads();
    if ((pl & ((1 << pin) - 1)) == 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            both[(pl >> pin) * wide + t.col + i] = c1[i];
            both[TH * 8 + (pl >> pin) * wide + t.col + i] = c2[i];
        }
    __syncthreads();
    for (int j = threadIdx.x; j < s.cn; j += TH) {
        float u = 0.0f, w = 0.0f;
        for (int r = 0; r < rows; ++r) u += both[r * wide + j], w += both[TH * 8 + r * wide + j];
        a.chan[((size_t)s.slot * a.chunks + s.chunk) * a.c + s.c0 + j] = make_float2(u, w);
    }
}

// The second launch of the backward in chunks.
template <typename T, int U, bool KEPT> __global__ __launch_bounds__(kThreads) void qblock_norm_dx_kernel(NormArgs a) {
    constexpr int F = 8 / U;
    const NormSeg s(a);
    const NormThread<U, kThreads> t(a, s);
    const int c = s.c0 + t.col;
    float bet[8];
    norm_channels(a.beta, c, t.n8, 0.0f, bet);
    for (long long sample = s.slot; sample < a.n; sample += a.slots) {
        float mean[F], rstd[F], ta[F], tx[F], scale[8];
        norm_channels(a.gamma, c, t.n8, 1.0f, scale);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const long long at = sample * a.groups + s.g0 + t.gi[f];
            mean[f] = a.mean[at];
            rstd[f] = a.rstd[at];
            const float2 x = a.avg[at];
            ta[f] = x.x;
            tx[f] = rstd[f] * (rstd[f] * x.y);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) scale[i] *= rstd[i / U];
        if (t.n8 <= 0) continue;
        const bool room = NormSeg::room(a, sample * a.hw + s.p1);
        NormWalk w(a, s.c0, sample * a.hw + s.p0, (uint32_t)t.p, t.col);
        for (int px = s.p0 + t.p; px < s.p1; px += 2 << a.pnl, w.at += 2 << a.pnl) {
            NormPair<T, U, KEPT> raw[2];
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (px + (r << a.pnl) < s.p1) raw[r].load(a, w, r, U == 8 ? 8 : t.n8, room);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int at = px + (r << a.pnl);
                if (at >= s.p1) continue;
                float g[8], x[8];
                raw[r].gradient(g);
                raw[r].input(w, x);
                norm_differences<U, F>(mean, x);
                norm_slopes(a.act, scale, bet, x, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = scale[i] * g[i] - (ta[i / U] + x[i] * tx[i / U]);
                block_store8<T>(reinterpret_cast<T *>(w.ptr<T>(static_cast<char *>(a.out), r)), g, U == 8 ? 8 : t.n8, a.stream);
            }
        }
    }
}

// dgamma and dbeta from `rows` partial sums a channel: 16 channels a workgroup, 64 rows at a time, four requested
// together.
template <int = 0>
__global__ __launch_bounds__(1024) void qblock_norm_param_kernel(const float2 *chan, int rows, int c, float *dgamma, float *dbeta) {
    __shared__ float2 sum[64][17];
    const int col = threadIdx.x & 15, j = blockIdx.x * 16 + col, r0 = threadIdx.x >> 4;
    float u = 0.0f, w = 0.0f;
    if (j < c)
        for (int q = r0; q < rows; q += 4096) {  // (64 of a thread's rows, and sums of these)
            float2 t = make_float2(0.0f, 0.0f);
            const int end = min(rows, q + 4096);
            for (int r = q; r < end; r += 256) {
                float2 x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = r + 64 * k < rows ? chan[(size_t)(r + 64 * k) * c + j] : make_float2(0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < 4; ++k) t.x += x[k].x, t.y += x[k].y;
            }
            u += t.x, w += t.y;
        }
    sum[r0][col] = make_float2(u, w);
    __syncthreads();
    // a wave joins a column
    const int k = threadIdx.x >> 6, to = blockIdx.x * 16 + k;
    float2 x = sum[threadIdx.x & 63][k];
    for (int b = 1; b < 64; b <<= 1) x.x += __shfl_xor(x.x, b), x.y += __shfl_xor(x.y, b);
    if ((threadIdx.x & 63) || to >= c) return;
    if (dbeta) dbeta[to] = x.x;
    if (dgamma) dgamma[to] = x.y;
}

}  // namespace ql
