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

#include "qdevice.h"

namespace ql {

enum HeadAct { HEAD_NONE = 0, HEAD_RELU = 1, HEAD_GELU = 2, HEAD_GELU_TANH = 3, HEAD_SILU = 4 };

__device__ __forceinline__ float head_act(int act, float z) {
    switch (act) {
        case HEAD_RELU: return z > 0.0f ? z : z == z ? 0.0f : z;  // (NaN stays NaN)
        case HEAD_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
        case HEAD_GELU_TANH: return 0.5f * z * (1.0f + tanhf(0.79788456f * (z + 0.044715f * z * z * z)));
        case HEAD_SILU: return z / (1.0f + expf(-z));
        default: return z;
    }
}

__device__ __forceinline__ float head_act_slope(int act, float z) {
    switch (act) {
        case HEAD_RELU: return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
        case HEAD_GELU: return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * expf(-0.5f * z * z) * 0.39894228f;
        case HEAD_GELU_TANH: {
            const float t = tanhf(0.79788456f * (z + 0.044715f * z * z * z)), u = 1.0f - t * t;
            // (u is 0 where the polynomial behind it may have overflowed)
            return 0.5f * (1.0f + t) + (u == 0.0f ? 0.0f : 0.5f * z * u * 0.79788456f * (1.0f + 0.134145f * z * z));
        }
        case HEAD_SILU: {
            const float s = 1.0f / (1.0f + expf(-z));
            return s * (1.0f + z * (1.0f - s));
        }
        default: return 1.0f;
    }
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
};

struct HeadGemmArgs {
    const void *a, *b;
    long long lda, ldb;  // row strides: of i (KM) or t (NAT)
    int I, J, R;
    HeadOut o;
};

template <typename T>
__device__ __forceinline__ void head_store(const HeadOut &o, int J, int i, int j, float acc) {
    if (o.b) acc += o.b[j];
    if (o.z) static_cast<T *>(o.z)[(size_t)i * J + j] = from_f32<T>(acc);
    float y = head_act(o.act, acc);
    if (o.r) y += to_f32<T>(static_cast<const T *>(o.r)[(size_t)i * o.ldr + j]);
    static_cast<T *>(o.c)[(size_t)i * o.ldc + j] = from_f32<T>(y);
}

// Any sizes and strides: 64 x 64 tiles of C, four waves with a 32 x 32 block each, 64 bytes
// of t a step through LDS (K-contiguous rows of 80 bytes), elements loaded one by one.
template <typename T, bool ANAT, bool BNAT>
__global__ __launch_bounds__(kThreads) void qhead_gemm_any_kernel(HeadGemmArgs g) {
    constexpr int KT = 64 / (int)sizeof(T), ROW = 80;
    __shared__ __attribute__((aligned(16))) char la[64 * ROW], lb[64 * ROW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
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

// The backward's start: dz = dy o act'(z) (dense, where asked for) and the column sums of the
// unrounded dz over `rpp` rows as partial sums [part][n], joined below in the order of parts.
template <typename T>
__global__ __launch_bounds__(kThreads) void qhead_dz_kernel(const T *dy, long long ldy, const T *z, int act, int m, int n,
                                                            int rpp, T *dz, float *part) {
    __shared__ float sum[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j = blockIdx.x * 64 + lane;
    const int begin = blockIdx.y * rpp, end = min(m, begin + rpp);
    float s = 0.0f;
    if (j < n)
        for (int i = begin + wave; i < end; i += 4) {
            float v = to_f32<T>(dy[(size_t)i * ldy + j]);
            if (act != HEAD_NONE) v *= head_act_slope(act, to_f32<T>(z[(size_t)i * n + j]));
            if (dz) dz[(size_t)i * n + j] = from_f32<T>(v);
            s += v;
        }
    sum[wave][lane] = s;
    __syncthreads();
    if (part && wave == 0 && j < n)
        part[(size_t)blockIdx.y * n + j] = sum[0][lane] + sum[1][lane] + sum[2][lane] + sum[3][lane];
}

template <int = 0>
__global__ __launch_bounds__(kThreads) void qhead_colsum_kernel(const float *part, int parts, int n, float *db) {
    const int j = blockIdx.x * kThreads + threadIdx.x;
    if (j >= n) return;
    float s = 0.0f;
    for (int p = 0; p < parts; ++p) s += part[(size_t)p * n + j];
    db[j] = s;
}

}  // namespace ql
