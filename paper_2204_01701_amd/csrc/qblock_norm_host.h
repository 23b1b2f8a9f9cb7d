// qblock_norm_host.h -- the group normalization's plan, and the launchers of its two directions.
#pragma once

#include "qblock_host.h"
#include "qblock_norm.h"

namespace ql {
namespace host {

inline int log2_up(long long v) {
    int b = 0;
    while ((1LL << b) < v) ++b;
    return b;
}

struct NormPlan {
    bool fused;
    int th, r, u;  // threads, pixels a thread, channels a thread takes as one
    int es;        // bytes of a value
    NormArgs a;    // the geometry
    size_t part_bytes, joined_bytes, chan_bytes;
    size_t bytes() const { return part_bytes + joined_bytes + chan_bytes; }
};

template <bool STATS> void launch_norm_join(const NormArgs &a, hipStream_t st) {
    const int slices = a.chunks * a.parts, lanes = std::min(64, 1 << log2_up(slices));
    hipLaunchKernelGGL((qblock_norm_join_kernel<STATS>), dim3(grid_1d((long long)a.n * a.groups * lanes)), dim3(kThreads), 0, st, a);
}

ql_status launch_norm_fwd(ql_dtype t, const NormPlan &p, const NormArgs &a, hipStream_t st);
// (instantiated for either type in a translation unit of its own)
template <typename T> void launch_norm_bwd_of(const NormPlan &p, const NormArgs &a, bool kept, hipStream_t st);

}  // namespace host
}  // namespace ql
