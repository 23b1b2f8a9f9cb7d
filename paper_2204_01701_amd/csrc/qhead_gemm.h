// qhead_gemm.h -- the first-order layer's kernels (include/qhead.h): matrix products with
// the epilogue z = acc + b, y = act(z) + r, and the elementwise start of the backward.
//
// The three products of a layer are one form, C[i, j] = sum_t A(i, t) B(j, t):
//   forward      A = x  (i = row,    t = input)    B = w  (j = output, t = input)
//   d input      A = dz (i = row,    t = output)   B = w  (j = input,  t = output)
//   d weight     A = dz (i = output, t = row)      B = x  (j = input,  t = row)
// An operand is stored either with t contiguous ("KM") or with its own index i or j
// contiguous ("NAT": w in the second, both in the third).
#pragma once

#include "qpipe.h"

namespace ql {

enum HeadAct { HEAD_NONE = 0, HEAD_RELU = 1, HEAD_GELU = 2, HEAD_GELU_TANH = 3, HEAD_SILU = 4 };

// The activations from exp2 and a reciprocal (each within an ulp or so): absolute errors of a few
// 1e-7 (1 + |z|), where the library functions' branches would cost a GEMM epilogue several times the
// instructions.  erf by the rational approximation 7.1.26 of Abramowitz and Stegun, Handbook of
// Mathematical Functions (absolute error 1.5e-7).
__device__ __forceinline__ float head_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }
__device__ __forceinline__ float head_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// Phi(z), and e = exp(-z^2 / 2) for the slope.
__device__ __forceinline__ float head_phi(float z, float &e) {
    const float x = fabsf(z) * 0.70710678118f;
    const float t = head_rcp(1.0f + 0.3275911f * x);
    e = head_exp(-0.5f * z * z);
    const float p = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    const float tail = 0.5f * p * e;  // Phi(-|z|)
    return z < 0.0f ? tail : 1.0f - tail;
}
__device__ __forceinline__ float head_sigmoid(float z) { return head_rcp(1.0f + head_exp(-z)); }

template <int ACT> __device__ __forceinline__ float head_act(float z) {
    if constexpr (ACT == HEAD_RELU) return z > 0.0f ? z : z == z ? 0.0f : z;  // (NaN stays NaN)
    if constexpr (ACT == HEAD_GELU) {
        float e;
        return z * head_phi(z, e);
    }
    // 0.5 (1 + tanh u) = sigmoid(2 u)
    if constexpr (ACT == HEAD_GELU_TANH) return z * head_sigmoid(z * (1.5957691216f + 0.0713548163f * z * z));
    if constexpr (ACT == HEAD_SILU) return z * head_sigmoid(z);
    return z;
}

template <int ACT> __device__ __forceinline__ float head_act_slope(float z) {
    if constexpr (ACT == HEAD_RELU) return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    if constexpr (ACT == HEAD_GELU) {
        float e;
        const float p = head_phi(z, e);
        return p + (e == 0.0f ? 0.0f : z * e * 0.39894228040f);
    }
    if constexpr (ACT == HEAD_GELU_TANH) {
        const float s = head_sigmoid(z * (1.5957691216f + 0.0713548163f * z * z)), u = s * (1.0f - s);
        // (u is 0 where the polynomial behind it may have overflowed)
        return s + (u == 0.0f ? 0.0f : z * u * (1.5957691216f + 0.2140644488f * z * z));
    }
    if constexpr (ACT == HEAD_SILU) {
        const float s = head_sigmoid(z);
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}

// N values at once: the choice among the activations is uniform and made once for them.
template <int N> __device__ __forceinline__ void head_acts(int act, float *v) {
#define HEAD_ALL(A)                                           \
    case A:                                                   \
        _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] = head_act<A>(v[e]); \
        break
    switch (act) {
        HEAD_ALL(HEAD_RELU);
        HEAD_ALL(HEAD_GELU);
        HEAD_ALL(HEAD_GELU_TANH);
        HEAD_ALL(HEAD_SILU);
        default: break;
    }
#undef HEAD_ALL
}
// v *= act'(z)
template <int N> __device__ __forceinline__ void head_slopes(int act, const float *z, float *v) {
#define HEAD_ALL(A)                                           \
    case A:                                                   \
        _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] *= head_act_slope<A>(z[e]); \
        break
    switch (act) {
        HEAD_ALL(HEAD_RELU);
        HEAD_ALL(HEAD_GELU);
        HEAD_ALL(HEAD_GELU_TANH);
        HEAD_ALL(HEAD_SILU);
        default: break;
    }
#undef HEAD_ALL
}

// Output side of a product: C (ldc), and for the forward the epilogue's operands.
struct HeadOut {
    void *c;  // y, dx or dw
    long long ldc;
    const float *b;
    const void *r;
    long long ldr;
    void *z;  // dense, I x J
    int act;
    bool c_f32;  // c is float, whatever T
};

struct HeadGemmArgs {
    const void *a, *b;
    long long lda, ldb;  // row strides: of i (KM) or t (NAT)
    int I, J, R;
    HeadOut o;
    int i0, j0;  // a launch's first row and column of C, where C takes more than one (few rows, any layout)
};

template <typename T>
__device__ __forceinline__ void head_store(const HeadOut &o, int J, int i, int j, float acc) {
    if (o.b) acc += o.b[j];
    if (o.z) static_cast<T *>(o.z)[(size_t)i * J + j] = from_f32<T>(acc);
    float y = acc;
    head_acts<1>(o.act, &y);
    if (o.r) y += to_f32<T>(static_cast<const T *>(o.r)[(size_t)i * o.ldr + j]);
    if (o.c_f32) static_cast<float *>(o.c)[(size_t)i * o.ldc + j] = y;
    else static_cast<T *>(o.c)[(size_t)i * o.ldc + j] = from_f32<T>(y);
}

// Any sizes and strides, for products too small to gain from copies into whole vectors, and none at all (R = 0):
// 64 x 64 tiles of C, four waves with a 32 x 32 block each, 64 bytes
// of t a step through LDS (K-contiguous rows of 80 bytes), elements loaded one by one.
template <typename T, bool ANAT, bool BNAT>
__global__ __launch_bounds__(kThreads) void qhead_gemm_any_kernel(HeadGemmArgs g) {
    constexpr int KT = 64 / (int)sizeof(T), ROW = 80;
    __shared__ __attribute__((aligned(16))) char la[64 * ROW], lb[64 * ROW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int i0 = g.i0 + blockIdx.x * 64, j0 = g.j0 + blockIdx.y * 64;
    const T *A = static_cast<const T *>(g.a), *B = static_cast<const T *>(g.b);
    f32x16_t acc = {};
    auto stage = [&](const T *p, long long ld, bool nat, int r0, int rows, int t0, char *l) {
        for (int e = tid; e < 64 * KT; e += kThreads) {
            const int row = nat ? e & 63 : e / KT, t = nat ? e >> 6 : e % KT;
            T v = 0;
            if (r0 + row < rows && t0 + t < g.R)
                v = nat ? p[(size_t)(t0 + t) * ld + (r0 + row)] : p[(size_t)(r0 + row) * ld + (t0 + t)];
            *reinterpret_cast<T *>(l + row * ROW + t * sizeof(T)) = v;
        }
    };
    for (int t0 = 0; t0 < g.R; t0 += KT) {
        stage(A, g.lda, ANAT, i0, g.I, t0, la);
        stage(B, g.ldb, BNAT, j0, g.J, t0, lb);
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const v4u a = *reinterpret_cast<const v4u *>(la + ((wave >> 1) * 32 + (lane & 31)) * ROW + c * 32 + (lane >> 5) * 16);
            const v4u b = *reinterpret_cast<const v4u *>(lb + ((wave & 1) * 32 + (lane & 31)) * ROW + c * 32 + (lane >> 5) * 16);
            mfma_chunk<T>(a, b, acc);
        }
        __syncthreads();
    }
    const int j = j0 + (wave & 1) * 32 + (lane & 31);
    if (j >= g.J) return;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int i = i0 + (wave >> 1) * 32 + 8 * (v / 4) + 4 * (lane >> 5) + v % 4;
        if (i < g.I) head_store<T>(g.o, g.J, i, j, acc[v]);
    }
}

// --- large products ----------------------------------------------------------------------
// A workgroup computes a BI x BJ tile of C from a ring of NS stages in LDS (qpipe.h), each 64 bytes
// of t deep: 32 bf16 or 16 fp32.  A stage's operand tiles are copied straight into LDS through
// buffer resources; a lane with nothing to load (a row past the matrix, t past its end) passes an
// offset past the buffer and gets zeros.  KM tiles are read as 16-byte fragments, NAT tiles
// transposed on the read (bf16) or element by element (fp32, whose MFMAs take four times as
// long as the reads).  The MFMA's rows are j and its columns i, so a lane holds four neighbours of a row of C.
//
// Bound by the matrix cores and LDS about alike: a 256 x 256 tile's 64-byte step is 1030 clocks of MFMA, 768 of
// fragment reads and 256 of copies.  Eight waves of 128 x 64 reach 1190 TFLOP/s at 8192^3 in bf16 (the library
// 1287) and 1160 in the weight gradient of 8192 x 2048 over 4096 rows; four waves of 128 x 128, which read a
// third less from LDS but run alone on their SIMDs, 1067.  fp32: 147 TFLOP/s (of 157), 128 x 128 tiles 127.
constexpr uint32_t kPastBuffer = 0x80000000u;  // (resources claim 2^31 - 1 bytes; the host keeps a tile's offsets below)

template <typename T> struct HeadStep {
    static constexpr int BK = 64 / (int)sizeof(T);
};

// One operand's part in the copies of a stage: BX rows of C's side, W waves.
template <typename T, bool NAT, int BX, int W> struct HeadSrc {
    static constexpr int NI = BX / (16 * W);               // instructions a wave issues per stage
    static constexpr int S16 = BX * (int)sizeof(T) / 16;   // 16-byte slots in a NAT row
    static_assert(BX % (16 * W) == 0, "whole instructions");
    const char *base;
    size_t step_bytes;
    uint32_t off[NI];
    int at[NI];  // KM: the byte of t within the stage (the same for all); NAT: its row

    __device__ __forceinline__ static int swz(int row) { return sizeof(T) == 2 ? nat_swz<S16>(row) : 0; }

    __device__ __forceinline__ HeadSrc(const void *p, long long ld, int x0, int X, int wave, int lane) {
        const size_t ldb = (size_t)ld * sizeof(T);
        if constexpr (NAT) {
            base = static_cast<const char *>(p) + (size_t)x0 * sizeof(T);
            step_bytes = HeadStep<T>::BK * ldb;
        } else {
            base = static_cast<const char *>(p) + (size_t)x0 * ldb;
            step_bytes = 64;
        }
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            const int q = wave * NI + n;
            if constexpr (NAT) {
                constexpr int RPI = 64 / S16;
                const int row = q * RPI + lane / S16, slot = (lane % S16) ^ swz(row);
                const bool ok = x0 + slot * Elem<T>::VEC < X;
                off[n] = ok ? (uint32_t)(row * ldb) + slot * 16 : kPastBuffer;
                at[n] = row;
            } else {
                const int row = q * 16 + (lane >> 2), col = km_fill_col(lane);
                off[n] = x0 + row < X ? (uint32_t)(row * ldb) + col * 16 : kPastBuffer;
                at[n] = col * 16;
            }
        }
    }
    // Copies the stage of K step s (left: what remains of t from there, in `at`'s units; 0 or less: nothing).
    __device__ __forceinline__ void issue(int s, int left, char *tile, int wave, DmaPart &part) const {
        const __amdgpu_buffer_rsrc_t rs = raw_rsrc(base + (size_t)s * step_bytes, 0x7fffffffu);
#pragma unroll
        for (int n = 0; n < NI; ++n)
            if (part.take()) dma16_buf(rs, at[n] < left ? off[n] : kPastBuffer, 0, tile + (wave * NI + n) * 1024);
    }
    __device__ __forceinline__ static int left_at(int R, int s) {
        return NAT ? R - s * HeadStep<T>::BK : (R - s * HeadStep<T>::BK) * (int)sizeof(T);
    }
    // The 32 x (32-byte chunk c) MFMA fragment at row x of the tile.
    __device__ __forceinline__ static v4u frag(const char *tile, int x, int c, int lane) {
        if constexpr (!NAT) return lds_read16(tile + km_off(x + (lane & 31), 2 * c + (lane >> 5)));
        else if constexpr (sizeof(T) == 2) return nat_frag_bf16<S16>(tile, 16 * c, x, lane);
        else {
            const char *p = tile + (8 * c + 4 * (lane >> 5)) * (BX * 4) + (x + (lane & 31)) * 4;
            v4u v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint32_t *>(p + i * BX * 4);
            return v;
        }
    }
};

typedef uint32_t v4u_row __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any element

// Eight neighbours of a row of C: epilogue and stores (`n` of them are inside the row).
template <typename T> __device__ __forceinline__ void head_store8(T *p, const float *v, int n) {
    if (n >= 8) {
#pragma unroll
        for (int h = 0; h < 8; h += Elem<T>::VEC) *reinterpret_cast<v4u_row *>(p + h) = vpack<T>(v + h);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = from_f32<T>(v[e]);
    }
}
template <typename T> __device__ __forceinline__ void head_load8(const T *p, float *v, int n) {
    if (n >= 8) {
#pragma unroll
        for (int h = 0; h < 8; h += Elem<T>::VEC) {
            const v4u x = *reinterpret_cast<const v4u_row *>(p + h);
#pragma unroll
            for (int e = 0; e < Elem<T>::VEC; ++e) v[h + e] = vget<T>(x, e);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? to_f32<T>(p[e]) : 0.0f;
    }
}
// r: the residual's raw bits, loaded beforehand, where eight of its elements are inside the row.
template <typename T> struct HeadRaw8 {
    v4u v[8 / Elem<T>::VEC];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int h = 0; h < 8 / Elem<T>::VEC; ++h) v[h] = *reinterpret_cast<const v4u_row *>(p + h * Elem<T>::VEC);
    }
    __device__ __forceinline__ float get(int e) const { return vget<T>(v[e / Elem<T>::VEC], e % Elem<T>::VEC); }
};
template <typename T>
__device__ __forceinline__ void head_epilogue8(const HeadOut &o, int J, int i, int j, float *v, const float *b,
                                               const HeadRaw8<T> &raw) {
    const int n = J - j;
    if (o.b) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += b[e];
    }
    if (o.z) head_store8<T>(static_cast<T *>(o.z) + (size_t)i * J + j, v, n);
    head_acts<8>(o.act, v);
    if (o.r) {
        if (n >= 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += raw.get(e);
        } else {
            const T *r = static_cast<const T *>(o.r) + (size_t)i * o.ldr + j;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) v[e] += to_f32<T>(r[e]);
        }
    }
    if (o.c_f32) head_store8<float>(static_cast<float *>(o.c) + (size_t)i * o.ldc + j, v, n);
    else head_store8<T>(static_cast<T *>(o.c) + (size_t)i * o.ldc + j, v, n);
}

struct HeadTileArgs {
    HeadGemmArgs g;
    int ti, tj, splits, per;  // tiles; K steps of a split
    float *part;              // splits x I x J, for splits > 1
};

// Logical tile of a workgroup: the workgroups of an XCD take neighbouring tiles, in bands of
// eight rows of tiles, so that they share operands in its L2.
__device__ __forceinline__ void head_tile(int bid, int ti, int tj, int &i, int &j) {
    const int band = bid / (8 * tj), rows = min(8, ti - band * 8), in = bid - band * 8 * tj;
    i = band * 8 + in % rows;
    j = in / rows;
}

template <int BI, int BJ, int WVI, int NS> constexpr int head_tile_lds() {
    const int ring = NS * (BI + BJ) * 64, stage = BI / WVI * (BJ * 4 + 16);
    return ring > stage ? ring : stage;
}

template <typename T, bool ANAT, bool BNAT, int BI, int BJ, int WVI, int WVJ, int NS, int WGS, int NI1>
__global__ __launch_bounds__(64 * WVI *WVJ, WGS *WVI *WVJ / 4) void qhead_gemm_kernel(HeadTileArgs a) {
    constexpr int W = WVI * WVJ, TH = 64 * W, WI = BI / WVI, WJ = BJ / WVJ, MI = WI / 32, MJ = WJ / 32;
    constexpr int STAGE = (BI + BJ) * 64, BK = HeadStep<T>::BK;
    typedef HeadSrc<T, ANAT, BI, W> SA;
    typedef HeadSrc<T, BNAT, BJ, W> SB;
    __shared__ __attribute__((aligned(16))) char lds[head_tile_lds<BI, BJ, WVI, NS>()];
    const int lane = threadIdx.x & 63, wave = wave_id(), wi = wave / WVJ, wj = wave - wi * WVJ;
    const HeadGemmArgs &g = a.g;
    int bid = xcd_remap(blockIdx.x, a.ti * a.tj * a.splits);
    const int split = bid / (a.ti * a.tj);
    int ti, tj;
    head_tile(bid - split * a.ti * a.tj, a.ti, a.tj, ti, tj);
    const int i0 = ti * BI, j0 = tj * BJ;
    const int steps = (g.R + BK - 1) / BK, begin = split * a.per, nst = min(a.per, steps - begin);
    const SA sa(g.a, g.lda, i0, g.I, wave, lane);
    const SB sb(g.b, g.ldb, j0, g.J, wave, lane);
    f32x16_t acc[MI][MJ];
#pragma unroll
    for (int x = 0; x < MI; ++x)
#pragma unroll
        for (int y = 0; y < MJ; ++y) acc[x][y] = f32x16_t{};
    v4u fa[2][MI], fb[2][MJ];
    auto issue = [&](int s, int slot, bool live, int lo, int hi) {
        char *st = lds + slot * STAGE;
        DmaPart part(lo, hi);
        sa.issue(s, live ? SA::left_at(g.R, s) : 0, st, wave, part);
        sb.issue(s, live ? SB::left_at(g.R, s) : 0, st + BI * 64, wave, part);
    };
    auto read = [&](int slot, int c, int buf) {
        const char *st = lds + slot * STAGE;
#pragma unroll
        for (int x = 0; x < MI; ++x) fa[buf][x] = SA::frag(st, wi * WI + 32 * x, c, lane);
#pragma unroll
        for (int y = 0; y < MJ; ++y) fb[buf][y] = SB::frag(st + BI * 64, wj * WJ + 32 * y, c, lane);
    };
    auto mma = [&](int buf) {
#pragma unroll
        for (int x = 0; x < MI; ++x)
#pragma unroll
            for (int y = 0; y < MJ; ++y) mfma_chunk<T>(fb[buf][y], fa[buf][x], acc[x][y]);
    };
    run_ring<NS, SA::NI + SB::NI, NI1>(nst, begin, issue, read, mma);
    // Epilogue, one row of waves at a time: the accumulators go to LDS as rows of C, and come back as
    // eight neighbours a thread, whose global accesses are whole lines.  A pass's residuals are
    // all requested before its hand-over through LDS: one at a time their latency was 21 us a tile.
    constexpr int ROW = BJ * 4 + 16, CG = BJ / 8, SWEEP = TH / CG, IT = WI / SWEEP;
    const int jc = (threadIdx.x % CG) * 8, j = j0 + jc, r0 = threadIdx.x / CG;
    const bool whole = a.splits == 1 && g.o.r && j + 8 <= g.J;
    float b[8] = {};
    if (g.o.b && a.splits == 1) head_load8<float>(g.o.b + j, b, g.J - j);
#pragma unroll
    for (int p = 0; p < WVI; ++p) {
        const int ip = i0 + p * WI + r0;
        HeadRaw8<T> raw[IT] = {};
        if (whole) {
#pragma unroll
            for (int q = 0; q < IT; ++q)
                if (ip + q * SWEEP < g.I) raw[q].load(static_cast<const T *>(g.o.r) + (size_t)(ip + q * SWEEP) * g.o.ldr + j);
        }
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
        if (j >= g.J) continue;
#pragma unroll
        for (int q = 0; q < IT; ++q) {
            const int i = ip + q * SWEEP;
            if (i >= g.I) continue;
            float v[8];
            const char *l = lds + (r0 + q * SWEEP) * ROW + jc * 4;
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const v4f t = *reinterpret_cast<const v4f *>(l + h * 4);
                v[h] = t[0], v[h + 1] = t[1], v[h + 2] = t[2], v[h + 3] = t[3];
            }
            if (a.splits > 1) head_store8<float>(a.part + ((size_t)split * g.I + i) * g.J + j, v, g.J - j);
            else head_epilogue8<T>(g.o, g.J, i, j, v, b, raw[q]);
        }
    }
}

// The splits' partial products, in their order, and the epilogue; the splits' loads are requested
// four at a time.  Bound by memory: two splits of 4096 x 2048 in 18 us (4.6 TB/s).
template <typename T>
__global__ __launch_bounds__(kThreads) void qhead_join_kernel(HeadTileArgs a) {
    const HeadGemmArgs &g = a.g;
    const int groups = (g.J + 7) / 8;
    const long long total = (long long)g.I * groups;
    const size_t stride = (size_t)g.I * g.J;
    for (long long q = (long long)blockIdx.x * kThreads + threadIdx.x; q < total; q += (long long)gridDim.x * kThreads) {
        const int i = (int)(q / groups), j = (int)(q - (long long)i * groups) * 8, n = g.J - j;
        const float *p = a.part + (size_t)i * g.J + j;
        float v[8] = {}, b[8] = {};
        HeadRaw8<T> raw = {};
        if (g.o.r && n >= 8) raw.load(static_cast<const T *>(g.o.r) + (size_t)i * g.o.ldr + j);
        if (g.o.b) head_load8<float>(g.o.b + j, b, n);
        for (int s = 0; s < a.splits; s += 4) {
            float u[4][8];
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (s + x < a.splits) head_load8<float>(p + (s + x) * stride, u[x], n);
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (s + x < a.splits) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += u[x][e];
                }
        }
        head_epilogue8<T>(g.o, g.J, i, j, v, b, raw);
    }
}

// --- few rows of x (serving: single tokens) -----------------------------------------------
// C for I <= 16 rows: bound by reading B (the weights) once.  A workgroup takes 16 rows of B (output
// columns); its eight waves share t, and each keeps eight 16-byte loads a lane in flight, straight into the
// operand layout of the 16 x 16 MFMA (whose rows are j, columns i), from any alignment.  The waves'
// partial products meet in LDS, in their order.  1 to 16 rows of 4096 onto 4096, bf16: 12 us a call, 33.6 MB
// (fp32: 24 to 27); 16 loads in flight a lane are no faster (the ramp of a launch is half of the time).
template <typename T> __device__ __forceinline__ void head_mfma16(const v4u &a, const v4u &b, v4f &acc) {
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), acc, 0, 0, 0);
    }
}

// 16 bytes of a row from element t on, zeros from R on.
template <typename T> __device__ __forceinline__ v4u head_row16(const T *p, int t, int R) {
    constexpr int VEC = Elem<T>::VEC;
    v4u v = {0u, 0u, 0u, 0u};
    if (t + VEC <= R) {
        v = *reinterpret_cast<const v4u_row *>(p + t);
    } else if (t < R) {
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = t + e < R ? to_f32<T>(p[t + e]) : 0.0f;
        v = vpack<T>(f);
    }
    return v;
}

template <typename T>
__global__ __launch_bounds__(512) void qhead_few_kernel(HeadGemmArgs g) {
    constexpr int W = 8, U = 8, STEP = 4 * Elem<T>::VEC;  // t of an MFMA: 32 bf16, 16 fp32
    __shared__ v4f part[W][64];
    const int lane = threadIdx.x & 63, wave = wave_id(), row = lane & 15, off = (lane >> 4) * Elem<T>::VEC;
    const int j0 = g.j0 + blockIdx.x * 16;
    const T *a = static_cast<const T *>(g.a) + (size_t)min(row, g.I - 1) * g.lda;
    const T *b = static_cast<const T *>(g.b) + (size_t)min(j0 + row, g.J - 1) * g.ldb;
    const int ra = row < g.I ? g.R : 0;  // (rows past I are zeros; columns past J are not stored)
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    // wave w takes steps w, w + 8, ...: the workgroup reads whole pieces of B's rows at a time
    for (int t0 = wave * STEP; t0 < g.R; t0 += U * W * STEP) {
        v4u fa[U], fb[U];
#pragma unroll
        for (int u = 0; u < U; ++u) fb[u] = head_row16<T>(b, t0 + u * W * STEP + off, g.R);
#pragma unroll
        for (int u = 0; u < U; ++u) fa[u] = head_row16<T>(a, t0 + u * W * STEP + off, ra);
#pragma unroll
        for (int u = 0; u < U; ++u) head_mfma16<T>(fb[u], fa[u], acc);
    }
    part[wave][lane] = acc;
    __syncthreads();
    const int i = threadIdx.x >> 4, j = j0 + (threadIdx.x & 15);  // (lane l holds column l % 16, rows 4 (l / 16) + v)
    if (threadIdx.x >= 256 || i >= g.I || j >= g.J) return;
    const int jr = threadIdx.x & 15;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += reinterpret_cast<const float *>(&part[w][(jr >> 2) * 16 + i])[jr & 3];
    head_store<T>(g.o, g.J, i, j, v);
}

// rows x cols at any stride and alignment -> rows of `out_cols` (whole 16-byte vectors), zeros behind.
template <typename T>
__global__ __launch_bounds__(kThreads) void qhead_pad_kernel(const T *p, long long ld, long long rows, int cols, int out_cols, T *out) {
    constexpr int VEC = Elem<T>::VEC;
    const int vecs = out_cols / VEC;
    for (long long q = (long long)blockIdx.x * kThreads + threadIdx.x; q < rows * vecs; q += (long long)gridDim.x * kThreads) {
        const long long i = q / vecs;
        const int j = (int)(q - i * vecs) * VEC;
        const T *src = p + (size_t)i * ld + j;
        v4u v;
        if (j + VEC <= cols) {
            v = *reinterpret_cast<const v4u_row *>(src);
        } else {
            float f[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = j + e < cols ? to_f32<T>(src[e]) : 0.0f;
            v = vpack<T>(f);
        }
        *reinterpret_cast<v4u *>(out + (size_t)i * out_cols + j) = v;
    }
}

// The backward's start: dz = dy o act'(z) (rows of ldd, where asked for) and the column sums of the
// unrounded dz over `rpp` rows as partial sums [part][n], joined below in the order of parts.
// In bf16 dz is rounded once, to be the operand of both products' bf16 MFMAs, as an activation's gradient
// is wherever it passes between two bf16 operators; kept in two halves it would double the products.  dx and
// dw are then off by 0.0023 (norms) where their own rounding to bf16 makes 0.0017.
// A workgroup takes 256 columns, eight a thread, eight rows at a time.  Bound by memory: 4096 x 8192, bf16,
// in 46 us (4.4 TB/s).
template <typename T>
__global__ __launch_bounds__(kThreads) void qhead_dz_kernel(const T *dy, long long ldy, const T *z, int act, int m, int n,
                                                            int rpp, T *dz, long long ldd, float *part) {
    __shared__ float sum[8][256 + 8];
    const int cg = threadIdx.x & 31, rg = threadIdx.x >> 5;
    const int j = blockIdx.x * 256 + cg * 8;
    const int begin = blockIdx.y * rpp, end = min(m, begin + rpp);
    float s[8] = {};
    if (j < n)
        for (int i0 = begin + rg; i0 < end; i0 += 16) {
            float v[2][8], u[2][8];
#pragma unroll
            for (int x = 0; x < 2; ++x) {  // (two rows requested together)
                const int i = i0 + 8 * x;
                if (i >= end) continue;
                head_load8<T>(dy + (size_t)i * ldy + j, v[x], n - j);
                if (act != HEAD_NONE) head_load8<T>(z + (size_t)i * n + j, u[x], n - j);
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int i = i0 + 8 * x;
                if (i >= end) continue;
                if (act != HEAD_NONE) head_slopes<8>(act, u[x], v[x]);
                // (elements behind the row's end loaded as 0 stay 0: a padded dz has zeros there)
                if (dz) head_store8<T>(dz + (size_t)i * ldd + j, v[x], (int)min(ldd - j, 8LL));
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += v[x][e];
            }
        }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[rg][cg * 8 + e] = s[e];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= n) return;
    float t = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) t += sum[r][threadIdx.x];
    part[(size_t)blockIdx.y * n + c] = t;
}

// db: 32 columns a workgroup, eight threads each; j0: the launch's first column.
template <int = 0>
__global__ __launch_bounds__(kThreads) void qhead_colsum_kernel(const float *part, int parts, int n, int j0, float *db) {
    __shared__ float sum[8][32];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, j = j0 + blockIdx.x * 32 + c;
    float s = 0.0f;
    if (j < n)
        for (int p = r; p < parts; p += 8) s += part[(size_t)p * n + j];
    sum[r][c] = s;
    __syncthreads();
    if (r || j >= n) return;
#pragma unroll
    for (int q = 1; q < 8; ++q) s += sum[q][c];
    db[j] = s;
}

}  // namespace ql
