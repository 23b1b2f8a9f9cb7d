// qblock_keep.h -- activations in 8 bits (include/qblock.h): blocks of 32 neighbours of a row
// as whole numbers of at most 127 and one power of two.
//
// A power of two rather than amax / 127 for the scale: x / 2^E is exact, so the rounding to q is
// the only one, no two implementations can disagree about it, and x8 = q 2^E needs 7 bits, which
// bf16 has, so a bf16 product takes the checkpoint as it stands.  It costs up to one bit of the
// step (a factor of 1.4 on average), of which blocks of 32 instead of 128, at the same 1/32 byte a
// value, give back a sixth (the largest magnitude of 32 normal values is 2.35 sigma on average, of 128 2.83).
#pragma once

#include "qblock_act.h"

namespace ql {

constexpr int kKeep = 32;          // values of a block
constexpr uint32_t kKeepNaN = 255;  // its exponent byte where it holds a NaN or an infinity

typedef uint32_t v2u_byte __attribute__((ext_vector_type(2), aligned(1)));  // 8 bytes at any address

// E + 127 from the bits of the block's largest magnitude: 127 * 2^E = 1.984375 * 2^(E + 6), so the exponent goes up by one
// where the fraction is above 0x7e0000.
__device__ __forceinline__ uint32_t keep_exponent(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return kKeepNaN;
    return (uint32_t)max((int)((amax_bits + 0x1ffffu) >> 23) - 6, 1);
}
// 2^E (e = 0: 0; e = 255: NaN, which its products with any q are), and 2^-E.
__device__ __forceinline__ float keep_scale(uint32_t e) { return __uint_as_float(e == kKeepNaN ? 0x7fc00000u : e << 23); }
__device__ __forceinline__ float keep_inverse(uint32_t e) { return __uint_as_float((254u - min(e, 253u)) << 23); }

__device__ __forceinline__ uint32_t keep_amax8(const float *v) {
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffffu);  // (NaN above infinity above numbers)
    return a;
}

// Four values as bytes: v 2^-E + 1.5 * 2^23 has v / 2^E, rounded half to even, in its low byte.
__device__ __forceinline__ uint32_t keep_bytes4(const float *v, float inv) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(__builtin_fmaf(v[i], inv, 12582912.0f));
    return __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u) | __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
}
__device__ __forceinline__ v2u keep_bytes8(float *v, uint32_t e) {
    if (e == kKeepNaN) return v2u{0u, 0u};
    const float inv = keep_inverse(e);
    if (e == 249u) {  // (64 * 2^122 would be an infinity)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fminf(fmaxf(v[i], -0x1.f8p127f), 0x1.f8p127f);
    }
    return v2u{keep_bytes4(v, inv), keep_bytes4(v + 4, inv)};
}

// n (up to 8) bytes at any address.
__device__ __forceinline__ void keep_put8(int8_t *p, const v2u &b, int n) {
    if (n >= 8) {
        *reinterpret_cast<v2u_byte *>(p) = b;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (int8_t)((i < 4 ? b.x : b.y) >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ v2u keep_get8(const int8_t *p, int n) {
    v2u b = {0u, 0u};
    if (n >= 8) {
        b = *reinterpret_cast<const v2u_byte *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) b[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    }
    return b;
}
__device__ __forceinline__ void keep_values8(const v2u &b, uint32_t e, float *v) {
    const float s = keep_scale(e);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(b[i >> 2] >> (8 * (i & 3))) * s;
}

// Eight values of one block (this lane's place in it: lane % 4; the block's other lanes are beside it, with zeros
// for values behind the row's end) to their bytes.  The first of the four lanes has e to store.
__device__ __forceinline__ v2u keep_pack8(float *v, uint32_t &e) {
    uint32_t a = keep_amax8(v);
    a = max(a, (uint32_t)__shfl_xor((int)a, 1));
    a = max(a, (uint32_t)__shfl_xor((int)a, 2));
    e = keep_exponent(a);
    return keep_bytes8(v, e);
}

struct KeepArgs {
    void *x;
    long long ld;
    int8_t *q;
    uint8_t *e;
    long long rows, cols;
    long long blocks;  // of a row
};

// (row, first column) of the lane's eight values: four neighbouring lanes a block.
__device__ __forceinline__ bool keep_place(const KeepArgs &a, long long at, long long &row, long long &blk, int &col8) {
    const long long b = at >> 2;
    if (a.rows == 1) row = 0, blk = b;
    else if (((a.rows * a.blocks) >> 32) == 0) row = (uint32_t)b / (uint32_t)a.blocks, blk = b - row * a.blocks;
    else row = b / a.blocks, blk = b - row * a.blocks;
    col8 = (int)(at & 3) * 8;
    return row < a.rows && blk * kKeep + col8 < a.cols;
}

// Bound by memory; eight values a lane, whose block's maximum takes two exchanges in registers.
template <typename T> __global__ __launch_bounds__(kThreads) void qblock_pack8_kernel(KeepArgs a) {
    const long long total = a.rows * a.blocks * 4, step = (long long)gridDim.x * kThreads;
    for (long long at = (long long)blockIdx.x * kThreads + threadIdx.x; at < total; at += step) {
        long long row, blk;
        int col8;
        const bool in = keep_place(a, at, row, blk, col8);
        const long long col = blk * kKeep + col8;
        const int n = in ? (int)min(a.cols - col, 8LL) : 0;
        float v[8] = {};
        if (n > 0) head_load8<T>(static_cast<const T *>(a.x) + row * a.ld + col, v, n);
        uint32_t e;
        const v2u b = keep_pack8(v, e);  // (a block's four lanes are all here: total is a multiple of four)
        if (n > 0) keep_put8(a.q + row * a.cols + col, b, n);
        if (col8 == 0) a.e[row * a.blocks + blk] = (uint8_t)e;
    }
}

template <typename T> __global__ __launch_bounds__(kThreads) void qblock_unpack8_kernel(KeepArgs a) {
    const long long total = a.rows * a.blocks * 4, step = (long long)gridDim.x * kThreads;
    for (long long at = (long long)blockIdx.x * kThreads + threadIdx.x; at < total; at += step) {
        long long row, blk;
        int col8;
        if (!keep_place(a, at, row, blk, col8)) continue;
        const long long col = blk * kKeep + col8;
        const int n = (int)min(a.cols - col, 8LL);
        float v[8];
        keep_values8(keep_get8(a.q + row * a.cols + col, n), a.e[row * a.blocks + blk], v);
        // (float's 32 bytes a lane go out as two halves of a line, which streamed took 45 us for 32768 x 1024, else 27)
        block_store8<T>(static_cast<T *>(a.x) + row * a.ld + col, v, n, sizeof(T) == 2);
    }
}

}  // namespace ql
