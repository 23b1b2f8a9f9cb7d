// qhead_rows.h -- kernels over rows of logits (include/qhead.h): softmax
// statistics with the entropy and the K largest values, and the distillation
// loss; both with their gradients.
//
// Mathematics.  With c = log2(e) / T, m the largest logit of what was read and
// d_j = (z_j - m) c, a row is reduced to
//     S = sum 2^d_j,     D = sum 2^d_j d_j,
// and two parts of a row are joined by shifting both to the common maximum:
// S -> 2^s S, D -> 2^s (D + s S) for s = (m_old - m_new) c.  Then
//     log p_j = ln2 d_j - ln S,   entropy = ln S - ln2 D / S.
// d is formed as a difference, then a product: folding m c into one constant
// would overflow for a row at the type's lowest value, whose softmax is uniform.
// m starts at the lowest finite value, so that -inf logits alone leave S = 0 (the
// mark of an empty row) and no difference of infinities is formed for them; NaN
// and +inf make S NaN by themselves.
//
// A row is read as 16-byte vectors from its first element, whatever its
// alignment (a row of an odd vocabulary starts anywhere; bf16 rows off a dword
// are read at four fifths of the rate, 4.3 against 5.1 TB/s at 32767 and 32768),
// and its last V mod (16 / size) elements one by one.
//
// All of it is bound by memory where rows are many and long: the statistics read at 5.1
// TB/s (4096 rows of 32768, bf16) to 5.7 (fp32), their gradients move 5.0 to 5.1, the
// distillation step 4.4 to 4.9 (4096 of 131072, bf16; 2048 of 32768, fp32), where a device copy
// moves 4.9.  Some 1000 rows of 50001 are read at 5.2 TB/s in fp32 (38 us) but at 3.6 in
// bf16 (28 us): four workgroups a CU, with nothing requested while a chunk is
// summed.  In a training step the same reads push the gradients written before them out of the
// memory-side cache: 59 us in fp32 (64 behind a plain fill of 200 MB, idle time in
// between or not), 36 in bf16; the gradient then finds its logits there (70 us, 87 by itself).
// Short rows are bound by their launch and their steps: 8192 of 1000, bf16, take 9 us, their gradient 12.
#pragma once

#include "qdevice.h"

namespace ql {

typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any element

constexpr float kHeadLowest = -3.402823466e+38f;
constexpr float kHeadFloor = -1e30f;  // stands for -inf in products with a 0 from the same exponent
// The same for a log probability, whose product with an upstream gradient comes first: below every one whose
// probability is not 0 in 32 bits (2^-149 over a sum of up to 2^31), and no more, so that h / T may reach 2e36.
constexpr float kHeadLowLogp = -128.0f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kHeadTopMax = 128;
constexpr int kHeadJoinKeys = 2048;  // alternatives of a row's parts together

__device__ __forceinline__ float head_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// --- one row as 16-byte vectors ------------------------------------------------
template <typename T> struct HeadRow {
    static constexpr int VEC = Elem<T>::VEC;
    const T *p;
    int V, nfull, nvec;  // elements, whole vectors, vectors with the partial one
    __device__ __forceinline__ HeadRow(const T *row, int v) : p(row), V(v), nfull(v / VEC), nvec((v - 1) / VEC + 1) {}
    __device__ __forceinline__ v4u load(int j) const { return *reinterpret_cast<const v4u_any *>(p + (size_t)j * VEC); }
    // The vector behind the whole ones, -inf past the row's end.
    __device__ __forceinline__ v4u partial() const {
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const size_t i = (size_t)nfull * VEC + e;
            f[e] = i < (size_t)V ? to_f32<T>(p[i]) : -__builtin_inff();
        }
        return vpack<T>(f);
    }
};

template <typename T> __device__ __forceinline__ v4u head_neg_inf() {
    const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    return v4u{w, w, w, w};
}

// r[u] = vector first + u * step + (this thread), -inf from `end` on.
template <typename T, int U>
__device__ __forceinline__ void head_load(const HeadRow<T> &row, int first, int step, int tid, int end, v4u (&r)[U]) {
    const int whole = min(end, row.nfull);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = first + u * step + tid;
        r[u] = head_neg_inf<T>();
        if (j < whole) r[u] = row.load(j);
    }
    if (end > row.nfull && first + U * step > row.nfull) {
        const v4u t = row.partial();
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + u * step + tid == row.nfull) r[u] = t;
    }
}

// z / T - m / T: halved around the difference, which would overflow between values at both
// ends of the type (their quotient by T need not).
__device__ __forceinline__ float head_scaled_diff(float z, float m, float inv_t) {
    return (0.5f * z - 0.5f * m) * inv_t * 2.0f;
}

// --- running sums ----------------------------------------------------------------
// s1 is the sum at T = 1 beside the one at T (distillation with labels), d the
// entropy's; each kernel keeps those it needs.
struct HeadSums {
    float m, s, d, s1;
};
__device__ __forceinline__ HeadSums head_start() { return {kHeadLowest, 0.0f, 0.0f, 0.0f}; }

// Shift `a` to the maximum m >= a.m.
template <bool ENT, bool TWO>
__device__ __forceinline__ void head_shift(HeadSums &a, float m, float c) {
    const float x = fmaxf((a.m - m) * c, kHeadFloor), f = head_exp2(x);
    if constexpr (ENT) a.d = f * (a.d + x * a.s);
    a.s *= f;
    if constexpr (TWO) a.s1 *= head_exp2((a.m - m) * kLog2e);
    a.m = m;
}

template <bool ENT, bool TWO>
__device__ __forceinline__ void head_join(HeadSums &a, HeadSums b, float c) {
    const float m = fmaxf(a.m, b.m);
    head_shift<ENT, TWO>(a, m, c);
    head_shift<ENT, TWO>(b, m, c);
    a.s += b.s;
    if constexpr (ENT) a.d += b.d;
    if constexpr (TWO) a.s1 += b.s1;
}

// The sums of U vectors held in registers; returns their maximum.
template <typename T, int U, bool ENT, bool TWO>
__device__ __forceinline__ float head_accumulate(HeadSums &a, v4u (&r)[U], float c) {
    constexpr int VEC = Elem<T>::VEC;
    float top = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = fmaxf(top, vget<T>(r[u], e));
    if (top > a.m) head_shift<ENT, TWO>(a, top, c);
    if constexpr (U >= 8) {
        // (unpacked anew: kept from above, the values of so many vectors would fill the registers)
#pragma unroll
        for (int u = 0; u < U; ++u) asm volatile("" : "+v"(r[u]));
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float x = vget<T>(r[u], e) - a.m, d = x * c, p = head_exp2(d);
            a.s += p;
            if constexpr (ENT) a.d += p * fmaxf(d, kHeadFloor);
            if constexpr (TWO) a.s1 += head_exp2(x * kLog2e);
            if constexpr (U >= 8)
                if (e == VEC - 1) __builtin_amdgcn_sched_barrier(0);  // (one vector's values at a time)
        }
    return top;
}

template <bool ENT, bool TWO> __device__ __forceinline__ HeadSums head_wave_join(HeadSums a, float c) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        HeadSums b = head_start();
        b.m = __shfl_xor(a.m, o);
        b.s = __shfl_xor(a.s, o);
        if constexpr (ENT) b.d = __shfl_xor(a.d, o);
        if constexpr (TWO) b.s1 = __shfl_xor(a.s1, o);
        head_join<ENT, TWO>(a, b, c);
    }
    return a;
}

// Join of at most 64 parts of a row, in every wave.
constexpr int kHeadMaxSplits = 64;
template <bool ENT, bool TWO>
__device__ __forceinline__ HeadSums head_join_parts(const HeadSums *part, int n, float c) {
    HeadSums a = head_start();
    const int lane = threadIdx.x & 63;
    if (lane < n) a = part[lane];
    return head_wave_join<ENT, TWO>(a, c);
}

// Join over the workgroup, in a fixed order; every thread gets the result.
template <int TH, bool ENT, bool TWO>
__device__ __forceinline__ HeadSums head_block_join(HeadSums a, float c, HeadSums *lds) {
    a = head_wave_join<ENT, TWO>(a, c);
    if constexpr (TH == 64) return a;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    a = lds[0];
#pragma unroll
    for (int w = 1; w < TH / 64; ++w) head_join<ENT, TWO>(a, lds[w], c);
    return a;
}

// --- the K largest ------------------------------------------------------------------
// An element's key: its value's bits in an order that unsigned integers share, over the
// complement of its index, so that equal values rank by the lower index and no two
// keys are equal.  -0 counts as 0.  NaN ranks behind every value; 0 is no element.
constexpr uint32_t kKeyNaN = 1u, kKeyNegInf = 0x007fffffu;

__device__ __forceinline__ uint32_t head_key(float z) {
    if (!(z == z)) return kKeyNaN;
    const uint32_t u = __float_as_uint(z + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float head_unkey(uint32_t k) {
    if (k < kKeyNegInf) return __builtin_nanf("");
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t head_key64(uint32_t k, int i) { return (uint64_t)k << 32 | (uint32_t)~i; }

// Candidates (and blocks that may hold some) a workgroup can list.
constexpr int head_cap(int threads) { return threads == 64 ? 512 : 1024; }
constexpr int kHeadGroups = 16;   // blocks a thread's share of a row is divided into at most

template <int TH> struct HeadTopLds {
    static constexpr int CAP = head_cap(TH);
    union {
        uint16_t top[kHeadGroups * TH];  // the upper halves of the blocks' largest keys, while the row is read
        uint64_t buf[CAP];               // candidates
    };
    uint64_t best[kHeadTopMax];          // the K best in order
    uint16_t block[CAP];
    int hist[256], pick[2];
    int wave[TH / 64];
    int n, blocks;                       // candidates and blocks found (those past CAP were not kept)
};

// The largest key of 16 bits that at least j of the wave's 64 x N keys reach: bits are set from the top
// while j stay at or above.  (The lower 16 bits stay 0: bf16 values have none, and for fp32 a bound
// slightly too low only costs candidates.)
template <int N> __device__ __forceinline__ uint32_t head_wave_kth(const uint32_t (&key)[N], int j) {
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t up = t | 1u << bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__ballot(key[i] >= up));
        if (n >= j) t = up;
    }
    return t;
}

// First wave: the bin at which the counts of hist[0 .. 255], taken in order, reach j (pick[0], -1: they do
// not), and how many of j are left for it (pick[1]).
__device__ __forceinline__ void head_hist_pick(const int *hist, int j, int *pick) {
    const int lane = threadIdx.x;
    int c[4], sum = 0;  // this lane's four bins
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += c[i] = hist[4 * lane + i];
    int x = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    int before = x - sum;
    if (lane == 63 && x < j) pick[0] = -1;
    if (before < j && x >= j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (before < j && before + c[i] >= j) {
                pick[0] = 4 * lane + i;
                pick[1] = j - before;
            }
            before += c[i];
        }
    }
}

// The same over the workgroup, exactly, by histograms of the keys' upper halves.  (Each wave's share of j, and
// the least of their answers, took no barriers but bounded rows whose large values lie together, sorted
// ones say, by far too little: 1333 us for 4096 rows of 32768, K = 64.)  First by distance from the largest key, where
// 256 bins are two octaves of bf16 and spread the counts; where fewer than j are so near, by the upper
// byte, then the lower.  Keys of 0 are none; 0 if there are fewer than j.
template <int TH, int N>
__device__ __forceinline__ uint32_t head_block_kth(const uint32_t (&key)[N], int j, int *hist, int *pick, int *wave) {
    if constexpr (TH == 64) return head_wave_kth(key, j);
    const int tid = threadIdx.x;
    int most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) most = max(most, (int)(key[i] >> 16));
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) most = max(most, __shfl_xor(most, o));
    if (tid < 256) hist[tid] = 0;
    if ((tid & 63) == 0) wave[tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) most = max(most, wave[w]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int d = most - (int)(key[i] >> 16);
        if (key[i] != 0 && d < 256) atomicAdd(&hist[d], 1);
    }
    __syncthreads();
    if (tid < 64) head_hist_pick(hist, j, pick);
    __syncthreads();
    if (pick[0] >= 0) return (uint32_t)(most - pick[0]) << 16;
    uint32_t t = 0;
#pragma unroll 1
    for (int shift = 24; shift >= 16; shift -= 8) {
        __syncthreads();
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (key[i] != 0 && (shift == 24 || key[i] >> 24 == t >> 24)) atomicAdd(&hist[255 - (key[i] >> shift & 255)], 1);
        __syncthreads();
        if (tid < 64) head_hist_pick(hist, j, pick);
        __syncthreads();
        if (pick[0] < 0) return 0;  // (the same for all)
        j = pick[1];
        t |= (uint32_t)(255 - pick[0]) << shift;
    }
    return t;
}

// Where this thread's `v` items go in a list of *n: the wave's sum is added once.
__device__ __forceinline__ int head_append(int v, int *n) {
    const int lane = threadIdx.x & 63;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    int at = 0;
    if (lane == 63 && x) at = atomicAdd(n, x);
    return __shfl(at, 63) + x - v;
}

// best: the K largest of the m keys, in order, by counting the larger ones of each.
template <int TH> __device__ __forceinline__ void head_rank(const uint64_t *keys, int m, uint64_t *best, int K) {
    for (int i = threadIdx.x; i < m; i += TH) {
        const uint64_t k = keys[i];
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < m; ++j) above += keys[j] > k ? 1 : 0;
        if (above < K) best[above] = k;
    }
    __syncthreads();
}

// Exclusive prefix of v over the workgroup's threads, and the total.
template <int TH> __device__ __forceinline__ int head_prefix(int v, int &total, int *lds) {
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if ((int)(threadIdx.x & 63) >= o) x += y;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) {
        if (w < (int)(threadIdx.x >> 6)) before += lds[w];
        total += lds[w];
    }
    return before + x - v;
}

// The elements of vector j of a row whose key is at least kmin, as a bit mask; none from vector `end` on.
template <typename T> __device__ __forceinline__ uint32_t head_mask(const HeadRow<T> &z, int j, int end, uint32_t kmin, v4u &r) {
    constexpr int VEC = Elem<T>::VEC;
    if (j >= end) return 0;
    r = j < z.nfull ? z.load(j) : z.partial();
    uint32_t mask = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) mask |= head_key(vget<T>(r, e)) >= kmin ? 1u << e : 0u;
    return j < z.nfull ? mask : mask & ((1u << (z.V - z.nfull * VEC)) - 1);
}
template <typename T> __device__ __forceinline__ uint32_t head_mask(const HeadRow<T> &z, int j, int end, uint32_t kmin) {
    v4u r;
    return head_mask<T>(z, j, end, kmin, r);
}

// The key of element e of a vector, e known at run time only.
template <typename T> __device__ __forceinline__ uint64_t head_key_of(const v4u &r, int e, int i) {
    const int d = sizeof(T) == 2 ? e >> 1 : e;
    const uint32_t w = d & 2 ? (d & 1 ? r.w : r.z) : (d & 1 ? r.y : r.x);
    return head_key64(head_key(sizeof(T) == 2 ? __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16) : __uint_as_float(w)), i);
}

// Too many candidates (equal values, mostly: a masked or constant row): the K-th largest key of the
// vectors [start, end) by bisection over re-reads, then what lies above it and the first ones equal
// to it in the order of their indices.  Leaves K candidates or more.
template <typename T, int TH>
__device__ __forceinline__ void head_top_crowd(HeadTopLds<TH> &s, const HeadRow<T> &z, int K, int start, int end, uint32_t least) {
    constexpr int VEC = Elem<T>::VEC;
    const int tid = threadIdx.x;
    auto count = [&](uint32_t k) {
        int n = 0, total;
#pragma unroll 1
        for (int j = start + tid; j < end; j += TH) n += __popc(head_mask<T>(z, j, end, k));
        head_prefix<TH>(n, total, s.wave);
        return total;
    };
    if (least <= kKeyNegInf) {  // a mask that leaves few: all of them are candidates
        const int finite = count(kKeyNegInf + 1);
        if (finite >= K && finite <= head_cap(TH)) {
            if (tid == 0) s.n = 0;
            __syncthreads();
#pragma unroll 1
            for (int j = start + tid; j < end; j += TH) {
                v4u r;
                uint32_t mine = head_mask<T>(z, j, end, kKeyNegInf + 1, r);
                if (!mine) continue;
                int to = atomicAdd(&s.n, __popc(mine));
                for (; mine; mine &= mine - 1, ++to) s.buf[to] = head_key_of<T>(r, __builtin_ctz(mine), j * VEC + __builtin_ctz(mine));
            }
            __syncthreads();
            return;
        }
    }
    uint32_t lo = least, hi = 0xffffffffu;  // count(lo) >= K > count(hi)
    if (count(lo + 1) < K) hi = lo + 1;     // rows of one value, and, in two more counts, masked ones
    if (hi - lo > 1 && lo < kKeyNegInf && count(kKeyNegInf + 1) < K) hi = kKeyNegInf + 1;
    if (hi - lo > 1 && hi == kKeyNegInf + 1 && count(kKeyNegInf) >= K) lo = kKeyNegInf;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (count(mid) >= K) lo = mid;
        else hi = mid;
    }
    int have = 0, total;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass)
#pragma unroll 1
        for (int first = start; first < end && have < K; first += TH) {  // (whole passes of TH vectors keep the order)
            const int j = first + tid;
            v4u r;
            uint32_t mine = head_mask<T>(z, j, end, pass ? lo : hi, r);
            if (pass) mine &= ~head_mask<T>(z, j, end, hi);
            int q = have + head_prefix<TH>(__popc(mine), total, s.wave);
            for (; mine && q < K; mine &= mine - 1, ++q) s.buf[q] = head_key_of<T>(r, __builtin_ctz(mine), j * VEC + __builtin_ctz(mine));
            have += total;
        }
    __syncthreads();
    if (tid == 0) s.n = min(have, K);
    __syncthreads();
}

// Candidates well over K (short rows, whose blocks bound little): bounded once more by themselves, since
// ranking takes n^2 steps (4000 rows of 600, K = 128, bf16: 189 us without).
template <int TH> __device__ __forceinline__ void head_top_prune(HeadTopLds<TH> &s, int K) {
    constexpr int PER = head_cap(TH) / TH;
    const int tid = threadIdx.x, n = s.n;
    uint64_t mine[PER];
    uint32_t key[PER];
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        mine[q] = q * TH + tid < n ? s.buf[q * TH + tid] : 0;
        key[q] = (uint32_t)(mine[q] >> 32);
    }
    const uint32_t least = head_block_kth<TH>(key, K, s.hist, s.pick, s.wave);
    __syncthreads();
    if (tid == 0) s.n = 0;
    __syncthreads();
    int kept = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) kept += mine[q] != 0 && key[q] >= least ? 1 : 0;
    int at = head_append(kept, &s.n);
#pragma unroll
    for (int q = 0; q < PER; ++q)
        if (mine[q] != 0 && key[q] >= least) s.buf[at++] = mine[q];
    __syncthreads();
}

// The K largest of vectors [start, end) of a row, into s.best.  While they were read, s.top got the upper
// halves of the largest keys of blocks of `rows` x one vector a thread; quarter[i]: the thread's largest
// value in blocks i mod 4.  These maxima belong to distinct elements, so the K-th largest of them bounds
// the row's K-th from below; only blocks that reach it are read again: little more than K of them,
// whatever the row's length.
template <typename T, int TH>
__device__ __forceinline__ void head_top(HeadTopLds<TH> &s, const HeadRow<T> &z, const float (&quarter)[4], int K, int start,
                                         int end, int rows) {
    constexpr int VEC = Elem<T>::VEC, CAP = head_cap(TH);
    const int tid = threadIdx.x;
    uint32_t key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)  // (a maximum of -inf may stand for nothing, or for NaN: it vouches for neither)
        key[i] = quarter[i] > -__builtin_inff() ? head_key(quarter[i]) : 0u;
    if (tid == 0) s.n = s.blocks = 0;
    const uint32_t least = head_block_kth<TH>(key, K, s.hist, s.pick, s.wave);
    if constexpr (TH == 64) __syncthreads();
    uint32_t mask = 0;
    for (int g = 0; start + g * rows * TH + tid < end; ++g) mask |= s.top[g * TH + tid] >= least >> 16 ? 1u << g : 0u;
    int at = head_append(__popc(mask), &s.blocks);
    for (; mask; mask &= mask - 1, ++at)
        if (at < CAP) s.block[at] = (uint16_t)(__builtin_ctz(mask) * TH + tid);
    __syncthreads();
    const int blocks = s.blocks;
    if (blocks <= CAP) {
        for (int q = tid; q < blocks * rows; q += TH) {
            const int b = s.block[q / rows], j = start + (b / TH * rows + q % rows) * TH + b % TH;
            v4u r;
            uint32_t mine = head_mask<T>(z, j, end, least, r);
            if (!mine) continue;
            int to = atomicAdd(&s.n, __popc(mine));
            for (; mine; mine &= mine - 1, ++to)
                if (to < CAP) s.buf[to] = head_key_of<T>(r, __builtin_ctz(mine), j * VEC + __builtin_ctz(mine));
        }
        __syncthreads();
    }
    if (blocks > CAP || s.n > CAP) head_top_crowd<T, TH>(s, z, K, start, end, least);
    if (s.n > K + K / 2 + 64) head_top_prune<TH>(s, K);
    head_rank<TH>(s.buf, s.n, s.best, K);
}

struct HeadLogprobArgs {
    const void *z;
    long long ld, row0;     // row0: the launch's first row
    int V, K, splits, per;  // per: vectors of a split
    float c, inv_t;
    const int64_t *target;
    float *logp, *entropy, *lse, *top_logp;
    int64_t *top_ids;
    float *stats;
    HeadSums *part;      // rows x splits
    uint64_t *part_top;  // rows x splits x K
};

// A row's target and its logit (0: none, or past the vocabulary), requested early.
struct HeadTarget {
    int64_t id;
    float z;
};
template <typename T> __device__ __forceinline__ HeadTarget head_target(const HeadLogprobArgs &a, long long row) {
    const int64_t id = a.target[row];
    return {id, id >= 0 && id < a.V ? to_f32<T>((static_cast<const T *>(a.z) + row * a.ld)[id]) : 0.0f};
}

// What a row's statistics say of it (whole workgroup; best: its K largest keys in order).
template <typename T, int TH>
__device__ __forceinline__ void head_logprobs_finish(const HeadLogprobArgs &a, long long row, const HeadSums &t,
                                                     const uint64_t *best, const HeadTarget &g) {
    const float ls = logf(t.s);  // -inf for an empty row
    const bool empty = t.s == 0.0f;
    if (threadIdx.x == 0) {
        float lp = 0.0f;
        if (g.id >= a.V) lp = __builtin_nanf("");
        else if (g.id >= 0) lp = empty ? -__builtin_inff() : head_scaled_diff(g.z, t.m, a.inv_t) - ls;
        a.logp[row] = lp;
        if (a.entropy) a.entropy[row] = empty ? 0.0f : ls - kLn2 * (t.d / t.s);
        if (a.lse) a.lse[row] = empty ? -__builtin_inff() : t.m * a.inv_t + ls;
        if (a.stats) {
            a.stats[2 * row] = t.m;
            a.stats[2 * row + 1] = t.s;
        }
    }
    for (int k = threadIdx.x; k < a.K; k += TH) {
        const uint64_t key = best[k];
        a.top_logp[row * a.K + k] =
            empty ? -__builtin_inff() : head_scaled_diff(head_unkey((uint32_t)(key >> 32)), t.m, a.inv_t) - ls;
        a.top_ids[row * a.K + k] = (int64_t)(uint32_t)~(uint32_t)key;
    }
}

// A workgroup per row, or per part of a row where rows are few: one pass for the sums and the blocks'
// maxima, then the K largest from the blocks that can hold them.  4096 rows of 32768, bf16: 52 us without
// alternatives, 60 with one, 72 with 64 (the blocks read again come from the memory-side cache,
// and ranking some 70 keys is most of the rest); keeping candidates chunk by chunk and ranking per
// chunk took 450, and held one workgroup a CU.
template <typename T, int TH, int U, bool TOP>
__global__ __launch_bounds__(TH) void qhead_logprobs_kernel(HeadLogprobArgs a) {
    __shared__ HeadSums sums[TH / 64];
    __shared__ HeadTopLds<TOP ? TH : 64> top;
    const int in = blockIdx.x / a.splits, sp = blockIdx.x - in * a.splits, tid = threadIdx.x;
    const long long row = a.row0 + in;
    const HeadRow<T> z(static_cast<const T *>(a.z) + row * a.ld, a.V);
    const int end = (int)min((long long)z.nvec, (long long)(sp + 1) * a.per);
    const HeadTarget g = head_target<T>(a, row);
    HeadSums t = head_start();
    const int start = sp * a.per;
    if constexpr (TOP) {
        const int steps = (end - start + U * TH - 1) / (U * TH), group = (steps + kHeadGroups - 1) / kHeadGroups;
        float quarter[4] = {-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
        for (int step = 0, b = 0; step < steps; step += group, ++b) {
            float here = -__builtin_inff();
            for (int i = step; i < min(step + group, steps); ++i) {
                v4u r[U];
                head_load<T, U>(z, start + i * U * TH, TH, tid, end, r);
                here = fmaxf(here, head_accumulate<T, U, true, false>(t, r, a.c));
            }
            // (NaN apart, which ranks behind everything and is found where all of a block counts)
            top.top[b * TH + tid] = (uint16_t)((here > -__builtin_inff() ? head_key(here) : kKeyNegInf) >> 16);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((b & 3) == i) quarter[i] = fmaxf(quarter[i], here);
        }
        head_top<T, TH>(top, z, quarter, a.K, start, end, group * U);
    } else {
        for (int first = start; first < end; first += U * TH) {
            v4u r[U];
            head_load<T, U>(z, first, TH, tid, end, r);
            head_accumulate<T, U, true, false>(t, r, a.c);
        }
    }
    t = head_block_join<TH, true, false>(t, a.c, sums);
    const uint64_t *best = nullptr;
    if constexpr (TOP) best = top.best;
    if (a.splits == 1) {
        head_logprobs_finish<T, TH>(a, row, t, best, g);
        return;
    }
    const long long at = row * a.splits + sp;
    if (tid == 0) a.part[at] = t;
    if constexpr (TOP)
        for (int k = tid; k < a.K; k += TH) a.part_top[at * a.K + k] = k < top.n ? best[k] : 0;
}

// Joins the parts of a row: what K of the parts' alternatives reach bounds the row's K-th from
// below, and only the alternatives that reach it are ranked.  Everything is requested from
// memory at once (one after the other, the latencies made up most of 15 us).
template <typename T>
__global__ __launch_bounds__(256) void qhead_logprobs_join_kernel(HeadLogprobArgs a) {
    extern __shared__ uint64_t cand[];  // splits x K
    __shared__ uint64_t best[kHeadTopMax];
    __shared__ int hist[256], pick[2], wave[4], n;
    const long long row = blockIdx.x;
    const int tid = threadIdx.x, K = a.K, keys = a.splits * K;
    constexpr int PER = kHeadJoinKeys / 256;
    uint64_t mine[PER];
#pragma unroll
    for (int q = 0; q < PER; ++q) mine[q] = tid + q * 256 < keys ? a.part_top[row * keys + tid + q * 256] : 0;
    const HeadTarget g = head_target<T>(a, row);
    const HeadSums t = head_join_parts<true, false>(a.part + row * a.splits, a.splits, a.c);
    if (K) {
        uint32_t key[PER];
#pragma unroll
        for (int q = 0; q < PER; ++q) key[q] = (uint32_t)(mine[q] >> 32);
        if (tid == 0) n = 0;
        const uint32_t least = head_block_kth<256>(key, K, hist, pick, wave);
        int kept = 0;
#pragma unroll
        for (int q = 0; q < PER; ++q) kept += mine[q] != 0 && key[q] >= least ? 1 : 0;
        int at = head_append(kept, &n);
#pragma unroll
        for (int q = 0; q < PER; ++q)
            if (mine[q] != 0 && key[q] >= least) cand[at++] = mine[q];
        __syncthreads();
        head_rank<256>(cand, n, best, K);
    }
    head_logprobs_finish<T, 256>(a, row, t, best, g);
}

// --- gradients --------------------------------------------------------------------------
// dz_j = A p_j + B p1_j + C p_j log p_j + (what the row's few ids add), with the
// probabilities formed from the row's m, S, S1.
struct HeadGrad {
    float m, c, a, b, e, is, is1, ls;
    bool zero;  // the row has no term: its gradient is 0 whatever the logits hold
};

template <bool ENT, bool TWO> __device__ __forceinline__ float head_grad_at(const HeadGrad &g, float z) {
    const float x = z - g.m, d = x * g.c, p = head_exp2(d) * g.is;
    float v = g.a;
    if constexpr (ENT) v += g.e * fmaxf(kLn2 * d - g.ls, kHeadLowLogp);
    v *= p;
    if constexpr (TWO) v += g.b * (head_exp2(x * kLog2e) * g.is1);
    return v;
}

// `more` is added at element `at` (-1: nowhere) by the thread that holds it.
template <typename T, int U, bool ENT, bool TWO>
__device__ __forceinline__ void head_grad_store(const HeadGrad &g, const HeadRow<T> &z, T *dz, const v4u (&r)[U], int first,
                                                int step, int tid, int end, int at = -1, float more = 0.0f) {
    constexpr int VEC = Elem<T>::VEC;
    const int whole = min(end, z.nfull), at_vec = at < 0 ? -1 : at / VEC;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = first + u * step + tid;
        if constexpr (U >= 8) __builtin_amdgcn_sched_barrier(0);  // (one vector's values at a time)
        if (j >= end) continue;
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = g.zero ? 0.0f : head_grad_at<ENT, TWO>(g, vget<T>(r[u], e));
        if (j == at_vec) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (e == at % VEC) f[e] += more;
        }
        T *o = dz + (size_t)j * VEC;
        if (j < whole) {
            *reinterpret_cast<v4u_any *>(o) = vpack<T>(f);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (j * (long long)VEC + e < z.V) o[e] = from_f32<T>(f[e]);
        }
    }
}

struct HeadLogprobGradArgs {
    const void *z;
    long long ld, row0;
    int V, splits, per;
    float c, inv_t;
    const int64_t *target;
    const float *stats, *entropy, *g, *h;
    void *dz;
};

template <typename T, int TH, int U, bool ENT>
__global__ __launch_bounds__(TH) void qhead_logprobs_grad_kernel(HeadLogprobGradArgs a) {
    const int in = blockIdx.x / a.splits, sp = blockIdx.x - in * a.splits, tid = threadIdx.x;
    const long long row = a.row0 + in;
    const HeadRow<T> z(static_cast<const T *>(a.z) + row * a.ld, a.V);
    T *dz = static_cast<T *>(a.dz) + row * a.V;
    const int begin = sp * a.per, end = (int)min((long long)z.nvec, (long long)(sp + 1) * a.per);
    const int64_t t = a.target[row];
    const bool given = t >= 0 && t < a.V;
    const float up = given ? a.g[row] : 0.0f, h = ENT ? a.h[row] : 0.0f, s = a.stats[2 * row + 1];
    HeadGrad g{};
    g.m = a.stats[2 * row];
    g.c = a.c;
    g.is = s == 0.0f ? 0.0f : 1.0f / s;
    g.ls = s == 0.0f ? 0.0f : logf(s);
    g.e = -h * a.inv_t;
    g.a = -up * a.inv_t + (ENT ? g.e * a.entropy[row] : 0.0f);
    g.zero = (up == 0.0f && h == 0.0f) || s == 0.0f;
    // The gradient may lie over the logits: an element is read and written by one thread only, the target's too.
    const int at = given && !g.zero ? (int)t : -1;
    const float more = up * a.inv_t;
    for (int first = begin; first < end; first += U * TH) {
        v4u r[U];
        head_load<T, U>(z, first, TH, tid, end, r);
        head_grad_store<T, U, ENT, false>(g, z, dz, r, first, TH, tid, end, at, more);
    }
}

// --- distillation ------------------------------------------------------------------------
struct HeadDistillArgs {
    const void *z;
    long long ld, row0;
    int V, K, splits, per;
    float c, temp, inv_t, alpha;
    const int64_t *ids;
    const void *tz;
    bool tz_f32;  // tz are float, whatever T
    const int64_t *label;
    const float *g;
    float *loss, *stats;  // stats: rows x 4, (m, S, S1, 0)
    HeadSums *part;
    void *dz;
};

// The few places of a row whose gradient has more than the probabilities: the teacher's K and, as
// place K, the label.  The first wave holds them, place lane + 64 i on a lane, so that they need no
// barriers of their own; what the other waves need of them goes through LDS with the row's sums.
constexpr int kHeadPlaces = (kHeadTopMax + 64) / 64;
struct HeadPlace {
    int id;          // -1: none
    float q;         // the teacher's logit, then the probability
    float zt, logq;  // student's logit, log q
};

template <int TH> struct HeadDistillLds {
    HeadSums sums[TH / 64];
    HeadPlace place[kHeadTopMax + 1];
    float has_q, has_l;  // the row has a teacher's term, a label's (0 or 1)
    uint8_t slot[2048];  // of the places' ids, the place written there last
};
__device__ __forceinline__ uint32_t head_slot(int id) { return (uint32_t)id * 2654435761u >> 21; }
static_assert(kHeadPlaces == 3 && kHeadTopMax < 256, "places of the first wave");

// In steps, each lane's places kept in LDS in between, so that the row can have the registers:
// the ids and the teacher's logits, the student's logits there (requests to memory without a branch on
// an id: place after place, their latencies cost 8 us a row of 128), and, once the row's gradient
// is under way, the softmax.  (First wave.)
struct HeadPlaceLoads {
    float zt[kHeadPlaces];
};
// Returns whether an id or the label is past the vocabulary.
template <typename T, int TH>
__device__ __forceinline__ bool head_places_load(const HeadDistillArgs &a, long long row, const T *z, HeadDistillLds<TH> &s,
                                                 HeadPlaceLoads &l) {
    int64_t id[kHeadPlaces];
    float t[kHeadPlaces];
#pragma unroll
    for (int i = 0; i < kHeadPlaces; ++i) {
        const int k = (int)threadIdx.x + 64 * i;
        id[i] = -1;
        t[i] = -__builtin_inff();
        if (k < a.K) {
            id[i] = a.ids[row * a.K + k];
            t[i] = a.tz_f32 ? static_cast<const float *>(a.tz)[row * a.K + k] : to_f32<T>(static_cast<const T *>(a.tz)[row * a.K + k]);
        } else if (k == a.K && a.label) {
            id[i] = a.label[row];
        }
    }
    bool wrong = false, label = false, some = false;
#pragma unroll
    for (int i = 0; i < kHeadPlaces; ++i) {
        const int k = (int)threadIdx.x + 64 * i;
        const bool in = id[i] >= 0 && id[i] < a.V;
        l.zt[i] = 0.0f;
        if (64 * i <= a.K) l.zt[i] = to_f32<T>(z[in ? id[i] : 0]);
        if (id[i] < 0) t[i] = -__builtin_inff();  // (an empty place, or one of probability 0)
        if (k <= a.K) s.place[k].id = in ? (int)id[i] : -1;
        if (k <= a.K) s.place[k].q = t[i];
        wrong = wrong || id[i] >= a.V;
        label = label || (k == a.K && in);
        some = some || t[i] != -__builtin_inff();
    }
    const bool has_l = __ballot(label) != 0, has_q = __ballot(some) != 0;
    if (threadIdx.x == 0) {
        s.has_q = has_q ? 1.0f : 0.0f;
        s.has_l = has_l ? 1.0f : 0.0f;
    }
    return __ballot(wrong) != 0;
}
template <int TH> __device__ __forceinline__ void head_places_keep(const HeadDistillArgs &a, const HeadPlaceLoads &l, HeadDistillLds<TH> &s) {
#pragma unroll
    for (int i = 0; i < kHeadPlaces; ++i)
        if ((int)threadIdx.x + 64 * i <= a.K) s.place[threadIdx.x + 64 * i].zt = l.zt[i];
}
template <int TH> __device__ __forceinline__ void head_places_softmax(const HeadDistillArgs &a, HeadDistillLds<TH> &s) {
    float t[kHeadPlaces], q[kHeadPlaces], most = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kHeadPlaces; ++i) {
        const int k = (int)threadIdx.x + 64 * i;
        t[i] = k <= a.K ? s.place[k].q : -__builtin_inff();
        most = fmaxf(most, t[i]);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kHeadPlaces; ++i) {
        const bool some = t[i] != -__builtin_inff();
        t[i] = (t[i] - most) * a.inv_t;
        q[i] = some ? expf(t[i]) : 0.0f;
        sum += q[i];
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    const float ls = logf(sum);
#pragma unroll
    for (int i = 0; i < kHeadPlaces; ++i) {
        const int k = (int)threadIdx.x + 64 * i;
        if (k > a.K) continue;
        s.place[k].q = sum != 0.0f ? q[i] / sum : 0.0f;
        s.place[k].logq = t[i] - ls;
    }
}

// The row's loss (first wave).
template <int TH>
__device__ __forceinline__ float head_distill_loss(const HeadDistillArgs &a, const HeadSums &t, bool wrong, const HeadDistillLds<TH> &s) {
    float v = 0.0f;
    const float ls = logf(t.s);
#pragma unroll
    for (int i = 0; i < kHeadPlaces; ++i) {
        const int k = (int)threadIdx.x + 64 * i;
        if (k > a.K) continue;
        const HeadPlace p = s.place[k];
        if (p.id < 0) continue;
        if (k < a.K) {
            const float lp = t.s == 0.0f ? -__builtin_inff() : head_scaled_diff(p.zt, t.m, a.inv_t) - ls;
            if (p.q != 0.0f) v += a.alpha * a.temp * a.temp * p.q * (p.logq - lp);
        } else {
            v += t.s1 == 0.0f ? __builtin_inff() : (1.0f - a.alpha) * (logf(t.s1) - head_scaled_diff(p.zt, t.m, 1.0f));
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    return wrong ? __builtin_nanf("") : v;
}

__device__ __forceinline__ HeadGrad head_distill_coef(const HeadDistillArgs &a, float has_q, float has_l, float m, float s,
                                                      float s1, float up) {
    HeadGrad g{};
    g.m = m;
    g.c = a.c;
    g.is = s == 0.0f ? 0.0f : 1.0f / s;
    g.is1 = s1 == 0.0f ? 0.0f : 1.0f / s1;
    g.a = up * a.alpha * a.temp * has_q;
    g.b = up * (1.0f - a.alpha) * has_l;
    g.zero = up == 0.0f || (has_q == 0.0f && has_l == 0.0f);
    return g;
}

// The places' own gradients, after the stream has written the row (first wave): each id is written by
// the first of the places that have it, with the sum of their parts.  Ids that occur twice are rare, so
// each place looks only whether its slot of a hash table was taken by another one (comparing each with all
// cost 9 us a row of 128), and those that lost theirs are compared with all.
template <typename T, int TH, bool TWO>
__device__ __forceinline__ void head_place_grads(const HeadDistillArgs &a, const HeadGrad &g, float up, T *dz, long long lo,
                                                 long long hi, HeadDistillLds<TH> &s) {
    float v[kHeadPlaces];
    int id[kHeadPlaces];
    __builtin_amdgcn_sched_barrier(0);
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        float q[kHeadPlaces];
        bool lost[kHeadPlaces], mine[kHeadPlaces];
#pragma unroll
        for (int i = 0; i < kHeadPlaces; ++i) {
            const int k = lane + 64 * i;
            id[i] = k < a.K ? s.place[k].id : -1;
            q[i] = k < a.K ? s.place[k].q : 0.0f;
            if (id[i] >= 0) s.slot[head_slot(id[i])] = (uint8_t)k;
        }
        wave_lds_sync();
#pragma unroll
        for (int i = 0; i < kHeadPlaces; ++i) {
            mine[i] = id[i] >= 0;
            lost[i] = mine[i] && s.slot[head_slot(id[i])] != lane + 64 * i;
        }
        const float own[kHeadPlaces] = {q[0], q[1], q[2]};
        for (;;) {
            int twice = -1;
#pragma unroll
            for (int i = 0; i < kHeadPlaces; ++i) {
                const uint64_t m = __ballot(lost[i]);
                if (m && twice < 0) twice = __builtin_amdgcn_readlane(id[i], __builtin_ctzll(m));
            }
            if (twice < 0) break;
            float sum = 0.0f;
            int first = -1;
#pragma unroll
            for (int i = 0; i < kHeadPlaces; ++i)
                for (uint64_t m = __ballot(id[i] == twice); m; m &= m - 1) {
                    const int l = __builtin_ctzll(m);
                    sum += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(own[i]), l));
                    if (first < 0) first = l + 64 * i;
                }
#pragma unroll
            for (int i = 0; i < kHeadPlaces; ++i)
                if (id[i] == twice) {
                    q[i] = sum;
                    mine[i] = lane + 64 * i == first;
                    lost[i] = false;
                }
        }
        const int label = s.place[a.K].id;
        bool among = false;  // (the label is one of the teacher's ids: it goes with that place)
#pragma unroll
        for (int i = 0; i < kHeadPlaces; ++i) among = among || __ballot(label >= 0 && id[i] == label) != 0;
#pragma unroll
        for (int i = 0; i < kHeadPlaces; ++i) {
            const int k = lane + 64 * i;
            if (k == a.K && !among) {
                id[i] = label;
                mine[i] = label >= 0;
            }
            v[i] = head_grad_at<false, TWO>(g, k <= a.K ? s.place[k].zt : 0.0f) - up * a.alpha * a.temp * q[i];
            if (label >= 0 && label == id[i]) v[i] -= up * (1.0f - a.alpha);
            if (!mine[i] || id[i] < lo || id[i] >= hi || g.zero) id[i] = -1;
        }
    }
    __syncthreads();
    if (threadIdx.x < 64) {
#pragma unroll
        for (int i = 0; i < kHeadPlaces; ++i)
            if (id[i] >= 0) dz[id[i]] = from_f32<T>(v[i]);
    }
}

__device__ __forceinline__ void head_distill_write(const HeadDistillArgs &a, long long row, const HeadSums &t, float loss) {
    a.loss[row] = loss;
    typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));  // (the caller's, at any element)
    if (a.stats) *reinterpret_cast<v4f_any *>(a.stats + 4 * row) = v4f_any{t.m, t.s, t.s1, 0.0f};
}

// One workgroup per row: the statistics, the loss and, for GRAD, the gradient.  HELD: the row fits the
// workgroup's registers, U vectors a thread, and is read once; else the gradient reads it again, from
// what the caches still hold of it.  (The values are unpacked anew for each pass over them and the places
// kept in LDS: with either in registers the rows of 16 vectors spilled, 600 us where this takes 440.)
template <typename T, int TH, int U, bool TWO, bool GRAD, bool HELD>
__global__ __launch_bounds__(TH, HELD &&U >= 8 ? 4 : 1) void qhead_distill_row_kernel(HeadDistillArgs a) {
    __shared__ HeadDistillLds<TH> s;
    const long long row = a.row0 + blockIdx.x;
    const int tid = threadIdx.x;
    const HeadRow<T> z(static_cast<const T *>(a.z) + row * a.ld, a.V);
    HeadSums t = head_start();
    v4u r[U];
    HeadPlaceLoads l;
    bool wrong = false;
    const float up = GRAD ? a.g[row] : 0.0f;
    head_load<T, U>(z, 0, TH, tid, z.nvec, r);
    if (tid < 64) {
        wrong = head_places_load<T, TH>(a, row, z.p, s, l);
        head_places_keep<TH>(a, l, s);
        head_places_softmax<TH>(a, s);
    }
    head_accumulate<T, U, false, TWO>(t, r, a.c);
    if constexpr (!HELD)
        for (int first = U * TH; first < z.nvec; first += U * TH) {
            head_load<T, U>(z, first, TH, tid, z.nvec, r);
            head_accumulate<T, U, false, TWO>(t, r, a.c);
        }
    t = head_block_join<TH, false, TWO>(t, a.c, s.sums);
    if constexpr (!TWO) t.s1 = t.s;
    if (tid < 64) {
        const float loss = head_distill_loss<TH>(a, t, wrong, s);
        if (tid == 0) head_distill_write(a, row, t, loss);
    }
    if constexpr (GRAD) {
        T *dz = static_cast<T *>(a.dz) + row * a.V;
        HeadGrad g = head_distill_coef(a, s.has_q, s.has_l, t.m, t.s, t.s1, up);
        if constexpr (!TWO) g.a += g.b;  // (T = 1, or no label: one set of probabilities)
        if constexpr (HELD) {
#pragma unroll
            for (int u = 0; u < U; ++u) asm volatile("" : "+v"(r[u]));  // (unpacked anew, as above)
            head_grad_store<T, U, false, TWO>(g, z, dz, r, 0, TH, tid, z.nvec);
        } else {
            for (int first = 0; first < z.nvec; first += U * TH) {
                head_load<T, U>(z, first, TH, tid, z.nvec, r);
                head_grad_store<T, U, false, TWO>(g, z, dz, r, first, TH, tid, z.nvec);
            }
        }
        head_place_grads<T, TH, TWO>(a, g, up, dz, 0, a.V, s);
    }
}

// Few rows: parts of rows on many workgroups, then a wave per row for the loss (64 rows of 131072, bf16, loss
// alone 12 us, a call's share included).
template <typename T, int TH, int U, bool TWO>
__global__ __launch_bounds__(TH) void qhead_distill_part_kernel(HeadDistillArgs a) {
    __shared__ HeadSums sums[TH / 64];
    const long long row = blockIdx.x / a.splits;
    const int sp = blockIdx.x - (int)row * a.splits;
    const HeadRow<T> z(static_cast<const T *>(a.z) + row * a.ld, a.V);
    const int end = (int)min((long long)z.nvec, (long long)(sp + 1) * a.per);
    HeadSums t = head_start();
    for (int first = sp * a.per; first < end; first += U * TH) {
        v4u r[U];
        head_load<T, U>(z, first, TH, threadIdx.x, end, r);
        head_accumulate<T, U, false, TWO>(t, r, a.c);
    }
    t = head_block_join<TH, false, TWO>(t, a.c, sums);
    if (threadIdx.x == 0) a.part[row * a.splits + sp] = t;
}

// One wave a row.
template <typename T, bool TWO>
__global__ __launch_bounds__(64) void qhead_distill_join_kernel(HeadDistillArgs a) {
    __shared__ HeadDistillLds<64> s;
    const long long row = blockIdx.x;
    HeadPlaceLoads l;
    const bool wrong = head_places_load<T, 64>(a, row, static_cast<const T *>(a.z) + row * a.ld, s, l);
    head_places_keep<64>(a, l, s);
    head_places_softmax<64>(a, s);
    HeadSums t = head_join_parts<false, TWO>(a.part + row * a.splits, a.splits, a.c);
    if constexpr (!TWO) t.s1 = t.s;
    const float loss = head_distill_loss<64>(a, t, wrong, s);
    if (threadIdx.x == 0) head_distill_write(a, row, t, loss);
}

template <typename T, int TH, int U, bool TWO>
__global__ __launch_bounds__(TH) void qhead_distill_grad_kernel(HeadDistillArgs a) {
    __shared__ HeadDistillLds<TH> s;
    const int in = blockIdx.x / a.splits, sp = blockIdx.x - in * a.splits, tid = threadIdx.x;
    const long long row = a.row0 + in;
    const HeadRow<T> z(static_cast<const T *>(a.z) + row * a.ld, a.V);
    const int begin = sp * a.per, end = (int)min((long long)z.nvec, (long long)(sp + 1) * a.per);
    T *dz = static_cast<T *>(a.dz) + row * a.V;
    const float up = a.g[row];
    const float *st = a.stats + 4 * row;
    v4u r[U];
    HeadPlaceLoads l;
    head_load<T, U>(z, begin, TH, tid, end, r);  // (in flight while the places are read)
    if (tid < 64) {
        head_places_load<T, TH>(a, row, z.p, s, l);
        head_places_keep<TH>(a, l, s);
        head_places_softmax<TH>(a, s);
    }
    __syncthreads();
    HeadGrad g = head_distill_coef(a, s.has_q, s.has_l, st[0], st[1], st[2], up);
    if constexpr (!TWO) g.a += g.b;
    for (int first = begin; first < end; first += U * TH) {
        if (first != begin) head_load<T, U>(z, first, TH, tid, end, r);
        head_grad_store<T, U, false, TWO>(g, z, dz, r, first, TH, tid, end);
    }
    head_place_grads<T, TH, TWO>(a, g, up, dz, (long long)begin * HeadRow<T>::VEC,
                                 min((long long)a.V, (long long)end * HeadRow<T>::VEC), s);
}

}  // namespace ql
