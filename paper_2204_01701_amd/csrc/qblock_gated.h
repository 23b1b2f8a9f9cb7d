// qblock_gated.h -- the gated layer's kernels (include/qblock.h): h = act(g) o u with g = x wg^T + bg
// and u = x wu^T + bu in one product, and the products of its backward.
//
// Three products on the LDS ring of qpipe.h, with the tiles and fragments of qhead_gemm.h:
//   GATED_FWD  C = x [wg; wu]^T.  A tile's columns are 32 of g, the same 32 of u, and so on, so that a
//              wave holds both factors of its part of h; they meet on their way through LDS.
//   GATED_DX   C = [dg du] [wg; wu]: one reduction over both halves; dg and du are padded to whole steps.
//   GATED_DW   C = [dg du]^T x: the rows of both weights' gradients, tiles of either in one launch.
#pragma once

#include "qblock_act.h"
#include "qblock_keep.h"

namespace ql {

enum GatedMode { GATED_FWD, GATED_DX, GATED_DW };

struct GatedOut {
    // forward
    const float *bg, *bu;
    void *h;
    long long ldh;
    void *z;  // 2 x I x n
    int8_t *q;
    uint8_t *e;
    int act;
    // backward: C, of which the rows from c_rows on are those of c1
    void *c0, *c1;
    bool c_f32;
};

struct GatedArgs {
    const void *a, *b0, *b1;
    long long lda, ldb;
    int I, J, R;  // FWD: rows, columns of h, inputs; DX: rows, inputs, outputs (of one half); DW: outputs (one half), inputs, rows
    int np;       // DX, DW: columns of a half of a, whole K steps
    GatedOut o;
    int ti, tj, splits, per, steps;
    float *part;  // splits x rows x columns of C, for splits > 1
};

// Eight neighbours of g and u: z, checkpoint, h.  n of them lie inside the row (none: the lane is here for its
// quad).
template <typename T>
__device__ __forceinline__ void gated_put(const GatedOut &o, int I, int J, int i, int j, int n, float *g, float *u) {
    if (o.z && n > 0) {
        T *z = static_cast<T *>(o.z) + (size_t)i * J + j;
        // (streamed: 8192 x 2048 -> 8192 with z, one set of weights in a row, in 493 us, 557 where the L2 keeps it; with three sets in
        // turn 543.  For h, which is half as much, and for the backward's outputs it makes no difference)
        block_store8<T>(z, g, n, true);
        block_store8<T>(z + (size_t)I * J, u, n, true);
    }
    if (o.q) {
        const int blocks = (J + kKeep - 1) / kKeep;
        auto keep = [&](const float *v, size_t row) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = k < n ? v[k] : 0.0f;
            uint32_t e;
            const v2u b = keep_pack8(x, e);
            if (n > 0) keep_put8(o.q + row * J + j, b, n);
            if (n > 0 && j % kKeep == 0) o.e[row * blocks + j / kKeep] = (uint8_t)e;
        };
        keep(g, i);
        keep(u, (size_t)I + i);
    }
    if (n <= 0) return;
    block_acts<8>(o.act, g);
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] *= u[k];
    head_store8<T>(static_cast<T *>(o.h) + (size_t)i * o.ldh + j, g, n);
}

// Eight neighbours of a row of C of the backward's products (rows of both halves counted through).
template <typename T, int MODE> __device__ __forceinline__ void gated_store(const GatedArgs &g, long long i, int j, const float *v) {
    void *c = g.o.c0;
    if (MODE == GATED_DW && i >= g.I) c = g.o.c1, i -= g.I;
    if (g.o.c_f32) head_store8<float>(static_cast<float *>(c) + (size_t)i * g.J + j, v, g.J - j);
    else head_store8<T>(static_cast<T *>(c) + (size_t)i * g.J + j, v, g.J - j);
}

// The forward's second operand: 64 rows of a tile are 32 rows of wg and the same 32 of wu.
template <typename T, int BX, int W> struct PairSrc {
    static constexpr int NI = BX / (16 * W);
    static_assert(NI == 2, "a wave copies 32 rows of one weight");
    const char *base;
    uint32_t off[NI];
    int at;
    __device__ __forceinline__ PairSrc(const void *p0, const void *p1, long long ld, int x0, int X, int wave, int lane) {
        const size_t ldb = (size_t)ld * sizeof(T);
        // (the choice is the wave's; told to the compiler, whose buffer resources have to be scalar)
        const uint64_t p = reinterpret_cast<uint64_t>(static_cast<const char *>(wave & 1 ? p1 : p0) + (size_t)x0 * ldb);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)p), hi = __builtin_amdgcn_readfirstlane((int)(p >> 32));
        base = reinterpret_cast<const char *>((uint64_t)hi << 32 | lo);
        const int col = km_fill_col(lane);
        at = col * 16;
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            const int q = wave * NI + n, row = (q >> 2) * 32 + (q & 1) * 16 + (lane >> 2);
            off[n] = x0 + row < X ? (uint32_t)(row * ldb) + col * 16 : kPastBuffer;
        }
    }
    __device__ __forceinline__ void issue(int s, int left, char *tile, int wave, DmaPart &part) const {
        const __amdgpu_buffer_rsrc_t rs = raw_rsrc(base + (size_t)s * 64, 0x7fffffffu);
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            if (part.take()) dma16_buf(rs, at < left ? off[n] : kPastBuffer, 0, tile + (wave * NI + n) * 1024);
        }
    }
    __device__ __forceinline__ static v4u frag(const char *tile, int x, int c, int lane) {
        return lds_read16(tile + km_off(x + (lane & 31), 2 * c + (lane >> 5)));
    }
};

// A workgroup's tile of a product: number `block` of its tiles and splits.
template <typename T, int MODE, int BI, int BJ, int WVI, int WVJ, int NS, int NI1>
__device__ __forceinline__ void gated_tile(const GatedArgs &g, int block, char *lds) {
    constexpr int W = WVI * WVJ, TH = 64 * W, WI = BI / WVI, WJ = BJ / WVJ, MI = WI / 32, MJ = WJ / 32;
    constexpr int STAGE = (BI + BJ) * 64, BK = HeadStep<T>::BK;
    static_assert(WJ == 64, "a wave's columns: 32 of g and 32 of u");
    typedef HeadSrc<T, MODE == GATED_DW, BI, W> SA;
    typedef HeadSrc<T, true, BJ, W> NatB;
    typedef PairSrc<T, BJ, W> PairB;
    constexpr int NIB = BJ / (16 * W);
    const int lane = threadIdx.x & 63, wave = wave_id(), wi = wave / WVJ, wj = wave - wi * WVJ;
    const int bid = xcd_remap(block, g.ti * g.tj * g.splits);
    const int split = bid / (g.ti * g.tj);
    int ti, tj;
    head_tile(bid - split * g.ti * g.tj, g.ti, g.tj, ti, tj);
    // (DW: the second half of the tiles' rows is that of wu's gradient)
    const bool second = MODE == GATED_DW && ti >= g.ti / 2;
    const int i0 = (second ? ti - g.ti / 2 : ti) * BI, j0 = tj * (MODE == GATED_FWD ? BJ / 2 : BJ);
    const int begin = split * g.per, nst = min(g.per, g.steps - begin);
    const SA sa(static_cast<const T *>(g.a) + (second ? g.np : 0), g.lda, i0, MODE == GATED_DW ? g.np : g.I, wave, lane);
    const PairB pb(g.b0, MODE == GATED_FWD ? g.b1 : g.b0, g.ldb, MODE == GATED_FWD ? j0 : 0, g.J, wave, lane);
    const NatB nb(g.b0, g.ldb, MODE == GATED_FWD ? 0 : j0, g.J, wave, lane);
    const char *nb1 = MODE == GATED_DX ? static_cast<const char *>(g.b1) + (nb.base - static_cast<const char *>(g.b0)) : nullptr;
    const int half = g.np / BK;  // (DX: K steps of a half)
    f32x16_t acc[MI][MJ];
#pragma unroll
    for (int x = 0; x < MI; ++x)
#pragma unroll
        for (int y = 0; y < MJ; ++y) acc[x][y] = f32x16_t{};
    v4u fa[2][MI], fb[2][MJ];
    auto issue = [&](int s, int slot, bool live, int lo, int hi) {
        char *st = lds + slot * STAGE;
        DmaPart part(lo, hi);
        if constexpr (MODE == GATED_FWD) {
            const int left = live ? SA::left_at(g.R, s) : 0;
            sa.issue(s, left, st, wave, part);
            pb.issue(s, left, st + BI * 64, wave, part);
        } else if constexpr (MODE == GATED_DX) {
            sa.issue(s, live ? 64 : 0, st, wave, part);  // (a's rows are whole steps)
            const bool up = s >= half;
            NatB b = nb;
            b.base = up ? nb1 : nb.base;
            const int t = up ? s - half : s;
            b.issue(t, live ? g.R - t * BK : 0, st + BI * 64, wave, part);
        } else {
            const int left = live ? g.R - s * BK : 0;
            sa.issue(s, left, st, wave, part);
            nb.issue(s, left, st + BI * 64, wave, part);
        }
    };
    auto read = [&](int slot, int c, int buf) {
        const char *st = lds + slot * STAGE;
#pragma unroll
        for (int x = 0; x < MI; ++x) fa[buf][x] = SA::frag(st, wi * WI + 32 * x, c, lane);
#pragma unroll
        for (int y = 0; y < MJ; ++y) {
            if constexpr (MODE == GATED_FWD) fb[buf][y] = PairB::frag(st + BI * 64, wj * WJ + 32 * y, c, lane);
            else fb[buf][y] = NatB::frag(st + BI * 64, wj * WJ + 32 * y, c, lane);
        }
    };
    auto mma = [&](int buf) {
#pragma unroll
        for (int x = 0; x < MI; ++x)
#pragma unroll
            for (int y = 0; y < MJ; ++y) mfma_chunk<T>(fb[buf][y], fa[buf][x], acc[x][y]);
    };
    run_ring<NS, SA::NI + NIB, NI1>(nst, begin, issue, read, mma);
    // Epilogue, one row of waves at a time, through LDS (as in qhead_gemm_kernel): eight neighbours a thread, in the
    // forward of g and, 32 columns on, of u.
    constexpr int ROW = BJ * 4 + 16, OJ = MODE == GATED_FWD ? BJ / 2 : BJ, CG = OJ / 8, SWEEP = TH / CG, IT = WI / SWEEP;
    static_assert(WI % SWEEP == 0, "whole sweeps");
    const int jc = (threadIdx.x % CG) * 8, j = j0 + jc, r0 = threadIdx.x / CG;
    const int lc = MODE == GATED_FWD ? (jc >> 5) * 64 + (jc & 31) : jc;
    float bg[8] = {}, bu[8] = {};
    if (MODE == GATED_FWD && g.splits == 1 && j < g.J) {
        if (g.o.bg) head_load8<float>(g.o.bg + j, bg, g.J - j);
        if (g.o.bu) head_load8<float>(g.o.bu + j, bu, g.J - j);
    }
#pragma unroll
    for (int p = 0; p < WVI; ++p) {
        lds_barrier();
        if (wi == p) {
#pragma unroll
            for (int x = 0; x < MI; ++x)
#pragma unroll
                for (int y = 0; y < MJ; ++y)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        *reinterpret_cast<v4f *>(lds + (32 * x + (lane & 31)) * ROW + (wj * WJ + 32 * y + 8 * v + 4 * (lane >> 5)) * 4) =
                            v4f{acc[x][y][4 * v], acc[x][y][4 * v + 1], acc[x][y][4 * v + 2], acc[x][y][4 * v + 3]};
        }
        lds_barrier();
#pragma unroll
        for (int q = 0; q < IT; ++q) {
            const int i = i0 + p * WI + r0 + q * SWEEP;
            if (i >= g.I) continue;
            const char *l = lds + (r0 + q * SWEEP) * ROW + lc * 4;
            float v[8], u[8];
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                const v4f t = *reinterpret_cast<const v4f *>(l + k * 4);
                v[k] = t[0], v[k + 1] = t[1], v[k + 2] = t[2], v[k + 3] = t[3];
                if constexpr (MODE == GATED_FWD) {
                    const v4f w = *reinterpret_cast<const v4f *>(l + 128 + k * 4);
                    u[k] = w[0], u[k + 1] = w[1], u[k + 2] = w[2], u[k + 3] = w[3];
                }
            }
            if constexpr (MODE == GATED_FWD) {
                if (g.splits > 1) {
                    if (j >= g.J) continue;
                    float *to = g.part + ((size_t)split * g.I + i) * 2 * g.J + j;
                    head_store8<float>(to, v, g.J - j);
                    head_store8<float>(to + g.J, u, g.J - j);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] += bg[k], u[k] += bu[k];
                    gated_put<T>(g.o, g.I, g.J, i, j, g.J - j, v, u);
                }
            } else {
                if (j >= g.J) continue;
                const long long row = second ? (long long)g.I + i : i;
                if (g.splits > 1)
                    head_store8<float>(g.part + ((size_t)split * (MODE == GATED_DW ? 2 : 1) * g.I + row) * g.J + j, v, g.J - j);
                else gated_store<T, MODE>(g, row, j, v);
            }
        }
    }
}

template <typename T, int MODE, int BI, int BJ, int WVI, int WVJ, int NS, int WGS, int NI1>
__global__ __launch_bounds__(64 * WVI *WVJ, WGS *WVI *WVJ / 4) void qblock_gated_kernel(GatedArgs g) {
    __shared__ __attribute__((aligned(16))) char lds[head_tile_lds<BI, BJ, WVI, NS>()];
    gated_tile<T, MODE, BI, BJ, WVI, WVJ, NS, NI1>(g, blockIdx.x, lds);
}

// Both products of the backward in one launch, those with the longer reduction first, so that the short ones fill up what
// their number leaves idle: 4096 x 2048 -> 8192 has 128 tiles of dx, 512 steps each, and 512 of the weights' gradients, 128
// each; together they are 512 steps for every CU, where dx by itself takes two splits and their join.
template <typename T, int BI, int BJ, int WVI, int WVJ, int NS, int WGS, int NI1>
__global__ __launch_bounds__(64 * WVI *WVJ, WGS *WVI *WVJ / 4) void qblock_gated_grads_kernel(GatedArgs dx, GatedArgs dw, int dx0, int dw0) {
    __shared__ __attribute__((aligned(16))) char lds[head_tile_lds<BI, BJ, WVI, NS>()];
    const int bid = blockIdx.x;
    if (bid >= dx0 && bid - dx0 < dx.ti * dx.tj) gated_tile<T, GATED_DX, BI, BJ, WVI, WVJ, NS, NI1>(dx, bid - dx0, lds);
    else gated_tile<T, GATED_DW, BI, BJ, WVI, WVJ, NS, NI1>(dw, bid - dw0, lds);
}

// Sum over the splits, in their order, of eight neighbours; four splits requested together.
__device__ __forceinline__ void gated_sum8(const float *p, size_t stride, int splits, int n, float *v) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    for (int s = 0; s < splits; s += 4) {
        float u[4][8];
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (s + x < splits) head_load8<float>(p + (s + x) * stride, u[x], n);
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (s + x < splits)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] += u[x][k];
    }
}

template <typename T, int MODE> __global__ __launch_bounds__(kThreads) void qblock_gated_join_kernel(GatedArgs g) {
    const int groups = (g.J + kKeep - 1) / kKeep * 4;  // (whole quads)
    const long long rows = MODE == GATED_DW ? 2LL * g.I : g.I, total = rows * groups;
    for (long long at = (long long)blockIdx.x * kThreads + threadIdx.x; at < total; at += (long long)gridDim.x * kThreads) {
        const long long i = at / groups;
        const int j = (int)(at - i * groups) * 8, n = g.J - j;
        float v[8] = {}, u[8] = {};
        if constexpr (MODE == GATED_FWD) {
            if (n > 0) {
                const float *p = g.part + (size_t)i * 2 * g.J + j;
                const size_t stride = (size_t)g.I * 2 * g.J;
                gated_sum8(p, stride, g.splits, n, v);
                gated_sum8(p + g.J, stride, g.splits, n, u);
                float b[8];
                if (g.o.bg) {
                    head_load8<float>(g.o.bg + j, b, n);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] += b[k];
                }
                if (g.o.bu) {
                    head_load8<float>(g.o.bu + j, b, n);
#pragma unroll
                    for (int k = 0; k < 8; ++k) u[k] += b[k];
                }
            }
            gated_put<T>(g.o, g.I, g.J, (int)i, j, n, v, u);
        } else if (n > 0) {
            gated_sum8(g.part + (size_t)i * g.J + j, (size_t)rows * g.J, g.splits, n, v);
            gated_store<T, MODE>(g, i, j, v);
        }
    }
}

// Up to 16 rows of x: bound by reading both weights once, from any layout (as qhead_few_kernel: 16 columns of h a
// workgroup, its eight waves share the reduction).
template <typename T> __global__ __launch_bounds__(512) void qblock_gated_few_kernel(GatedArgs g) {
    constexpr int W = 8, U = 4, STEP = 4 * Elem<T>::VEC;
    __shared__ v4f part[2][W][64];
    const int lane = threadIdx.x & 63, wave = wave_id(), row = lane & 15, off = (lane >> 4) * Elem<T>::VEC;
    const int j0 = blockIdx.x * 16;
    const T *a = static_cast<const T *>(g.a) + (size_t)min(row, g.I - 1) * g.lda;
    const size_t at = (size_t)min(j0 + row, g.J - 1) * g.ldb;
    const T *b0 = static_cast<const T *>(g.b0) + at, *b1 = static_cast<const T *>(g.b1) + at;
    const int ra = row < g.I ? g.R : 0;  // (rows past I are zeros; columns past J are not stored)
    v4f acc0 = {0.0f, 0.0f, 0.0f, 0.0f}, acc1 = acc0;
    struct Fragments {
        v4u a[U], f0[U], f1[U];
    } now, next;
    auto load = [&](Fragments &f, int t0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f.f0[u] = head_row16<T>(b0, t0 + u * STEP + off, g.R);
            f.f1[u] = head_row16<T>(b1, t0 + u * STEP + off, g.R);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) f.a[u] = head_row16<T>(a, t0 + u * STEP + off, ra);
    };
    auto multiply = [&](const Fragments &f) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            head_mfma16<T>(f.f0[u], f.a[u], acc0);
            head_mfma16<T>(f.f1[u], f.a[u], acc1);
        }
    };
    // (the next fragments are on their way while these are multiplied)
    constexpr int S = U * W * STEP;
    // (a wave's U steps lie side by side: 256 bytes of a row)
    load(now, wave * U * STEP);
    for (int t0 = wave * U * STEP; t0 < g.R; t0 += 2 * S) {
        load(next, t0 + S);
        multiply(now);
        load(now, t0 + 2 * S);
        multiply(next);
    }
    part[0][wave][lane] = acc0;
    part[1][wave][lane] = acc1;
    __syncthreads();
    const int i = threadIdx.x >> 4, jr = threadIdx.x & 15, j = j0 + jr;  // (lane l holds column l % 16, rows 4 (l / 16) + v)
    if (threadIdx.x >= 256 || i >= g.I || j >= g.J) return;
    float v[2] = {};
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
        for (int k = 0; k < 2; ++k) v[k] += reinterpret_cast<const float *>(&part[k][w][(jr >> 2) * 16 + i])[jr & 3];
    if (g.o.bg) v[0] += g.o.bg[j];
    if (g.o.bu) v[1] += g.o.bu[j];
    if (g.o.z) {
        T *z = static_cast<T *>(g.o.z) + (size_t)i * g.J + j;
        z[0] = from_f32<T>(v[0]);
        z[(size_t)g.I * g.J] = from_f32<T>(v[1]);
    }
    block_acts<1>(g.o.act, v);
    static_cast<T *>(g.o.h)[(size_t)i * g.o.ldh + j] = from_f32<T>(v[0] * v[1]);
}

// The backward's start: dg = dh o u o act'(g) and du = dh o act(g) from z or its checkpoint, as [row][half][np]
// with zeros behind each half (where dz is asked for), and their column sums over `rpp` rows, unrounded, as partial
// sums [part][2 n].  In bf16 dg and du are rounded once, to be operands of the products' MFMAs.
struct GatedDzArgs {
    const void *dh;
    long long ldh;
    const void *z;
    const int8_t *q;
    const uint8_t *e;
    int m, n, np, act, rpp;
    void *dz;
    float *part0, *part1;  // of dbg and dbu (either may be NULL)
    long long part_ld;
};

template <typename T, bool KEPT> __global__ __launch_bounds__(kThreads) void qblock_gated_dz_kernel(GatedDzArgs a) {
    __shared__ float sum[2][8][256 + 8];
    const int cg = threadIdx.x & 31, rg = threadIdx.x >> 5;
    const int j = blockIdx.x * 256 + cg * 8, n8 = a.n - j, blocks = (a.n + kKeep - 1) / kKeep;
    const int begin = blockIdx.y * a.rpp, end = min(a.m, begin + a.rpp);
    float s[2][8] = {};
    if (j < a.np)
        for (int i0 = begin + rg; i0 < end; i0 += 16) {
            float d[2][8], g[2][8], u[2][8];
#pragma unroll
            for (int x = 0; x < 2; ++x) {  // (two rows requested together)
                const int i = i0 + 8 * x;
                if (i >= end) continue;
                head_load8<T>(static_cast<const T *>(a.dh) + (size_t)i * a.ldh + j, d[x], n8);
                if constexpr (KEPT) {
                    if (n8 > 0) {
                        const size_t r0 = i, r1 = (size_t)a.m + i;
                        keep_values8(keep_get8(a.q + r0 * a.n + j, n8), a.e[r0 * blocks + j / kKeep], g[x]);
                        keep_values8(keep_get8(a.q + r1 * a.n + j, n8), a.e[r1 * blocks + j / kKeep], u[x]);
                    }
                } else {
                    const T *z = static_cast<const T *>(a.z) + (size_t)i * a.n + j;
                    head_load8<T>(z, g[x], n8);
                    head_load8<T>(z + (size_t)a.m * a.n, u[x], n8);
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int i = i0 + 8 * x;
                if (i >= end) continue;
                float dg[8], act[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    dg[k] = d[x][k] * u[x][k];
                    act[k] = g[x][k];
                }
                block_slopes<8>(a.act, g[x], dg);
                block_acts<8>(a.act, act);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    act[k] *= d[x][k];
                    if (k >= n8) dg[k] = act[k] = 0.0f;
                    s[0][k] += dg[k], s[1][k] += act[k];
                }
                if (a.dz) {
                    T *to = static_cast<T *>(a.dz) + (size_t)i * 2 * a.np + j;
                    head_store8<T>(to, dg, 8);  // (np is a multiple of 8)
                    head_store8<T>(to + a.np, act, 8);
                }
            }
        }
    if (!a.part0 && !a.part1) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[0][rg][cg * 8 + k] = s[0][k], sum[1][rg][cg * 8 + k] = s[1][k];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.n) return;
    float t0 = 0.0f, t1 = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) t0 += sum[0][r][threadIdx.x], t1 += sum[1][r][threadIdx.x];
    if (a.part0) a.part0[(size_t)blockIdx.y * a.part_ld + c] = t0;
    if (a.part1) a.part1[(size_t)blockIdx.y * a.part_ld + c] = t1;
}

// dbg and dbu from their partial sums: 32 columns a workgroup, eight threads each; a row of workgroups for either.
template <int = 0>
__global__ __launch_bounds__(kThreads) void qblock_gated_colsum_kernel(const float *part0, const float *part1, int parts, int n,
                                                                       float *dbg, float *dbu) {
    __shared__ float sum[8][32];
    const float *part = blockIdx.y ? part1 : part0;
    float *db = blockIdx.y ? dbu : dbg;
    if (!db) return;
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, j = blockIdx.x * 32 + c;
    float s = 0.0f;
    if (j < n)
        for (int p0 = r; p0 < parts; p0 += 512) {  // (64 parts, and sums of these)
            const int end = min(parts, p0 + 512);
            float t = 0.0f;
            for (int p = p0; p < end; p += 8) t += part[(size_t)p * n + j];
            s += t;
        }
    sum[r][c] = s;
    __syncthreads();
    if (r || j >= n) return;
#pragma unroll
    for (int q = 1; q < 8; ++q) s += sum[q][c];
    db[j] = s;
}

}  // namespace ql
