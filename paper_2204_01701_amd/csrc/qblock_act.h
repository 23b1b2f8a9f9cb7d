// qblock_act.h -- the activations of the block operators: those of qhead_gemm.h, with the error
// function's gelu in fewer instructions, since a pass over a map that evaluates it is bound by the
// vector ALU before it is by memory.
#pragma once

#include "qhead_gemm.h"

namespace ql {

// With x = |z| / sqrt 2, t = 1 / (1 + 0.3275911 x) and e = exp(-x^2), Phi(-|z|) = p(t) e for the polynomial p of Abramowitz and
// Stegun's 7.1.26 (halved).  As Phi(z) = 1 - Phi(-|z|) for z > 0,
//     gelu(z) = max(z, 0) - |z| Phi(-|z|),   gelu'(z) = [z > 0] + sign(z) e (|z| / sqrt(2 pi) - p).
// Where e is 0 the factors |z| are kept finite.  16 instructions and two of quarter rate for the slope (24 and two as
// written in qhead_gemm.h).
struct GeluParts {
    float e, p, a;
    __device__ __forceinline__ explicit GeluParts(float z) {
        const float u = z * 0.84932180028802f;  // sqrt(log2(e) / 2): e = 2^(-u^2)
        const float t = head_rcp(__builtin_fmaf(0.27273749f, fabsf(u), 1.0f));  // 0.3275911 / sqrt 2 / 0.8493218
        e = __builtin_amdgcn_exp2f(-u * u);
        p = t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f))));
        a = fminf(fabsf(z), 64.0f);
    }
};

template <int ACT> __device__ __forceinline__ float block_act(float z) {
    if constexpr (ACT == HEAD_GELU) {
        const GeluParts g(z);
        return fmaxf(z, 0.0f) - g.a * (g.p * g.e);
    }
    return head_act<ACT>(z);
}
template <int ACT> __device__ __forceinline__ float block_slope(float z) {
    if constexpr (ACT == HEAD_GELU) {
        const GeluParts g(z);
        const float y = g.e * __builtin_fmaf(0.39894228040f, g.a, -g.p);
        return z > 0.0f ? 1.0f + y : -y;
    }
    return head_act_slope<ACT>(z);
}

#define BLOCK_ALL(A, F, OP)                                                            \
    case A:                                                                            \
        _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] OP F<A>(z[e]);              \
        break
#define BLOCK_SWITCH(F, OP)              \
    switch (act) {                       \
        BLOCK_ALL(HEAD_RELU, F, OP);      \
        BLOCK_ALL(HEAD_GELU, F, OP);      \
        BLOCK_ALL(HEAD_GELU_TANH, F, OP); \
        BLOCK_ALL(HEAD_SILU, F, OP);      \
        default: break;                  \
    }
// N values at once (the choice among the activations is uniform and made once for them): v = act(v)
template <int N> __device__ __forceinline__ void block_acts(int act, float *v) {
    float *z = v;
    BLOCK_SWITCH(block_act, =)
}
// v *= act'(z)
template <int N> __device__ __forceinline__ void block_slopes(int act, const float *z, float *v) { BLOCK_SWITCH(block_slope, *=) }
#undef BLOCK_SWITCH
#undef BLOCK_ALL

// Eight neighbours stored as what is not read again (`stream`, uniform): they do not drive out of the L2 what the workgroups
// beside share, and a launch's stores do not queue behind its loads' lines.  For whole lines only: parts of them, written
// past the L2, reach memory one by one.
template <typename T> __device__ __forceinline__ void block_store8(T *p, const float *v, int n, bool stream) {
    if (stream && n >= 8) {
        // (without something of its own on either side the branch is merged with the other, and the hint is lost)
        asm volatile("" ::: "memory");
#pragma unroll
        for (int h = 0; h < 8; h += Elem<T>::VEC) __builtin_nontemporal_store(vpack<T>(v + h), reinterpret_cast<v4u_row *>(p + h));
        asm volatile("" ::: "memory");
    } else {
        head_store8<T>(p, v, n);
    }
}
}  // namespace ql
