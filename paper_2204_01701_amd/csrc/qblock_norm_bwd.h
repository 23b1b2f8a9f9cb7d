// qblock_norm_bwd.h -- launches of the group normalization's backward, one translation unit a type (they
// compile side by side).
#pragma once

#include "qblock_norm_host.h"

namespace ql {
namespace host {

template <typename T, int U, bool KEPT> void launch_norm_bwd_unit(const NormPlan &p, const NormArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)a.blocks), wg((unsigned)p.th);
    if (p.fused) {
        if (p.th == 512) hipLaunchKernelGGL((qblock_norm_bwd_kernel<T, 8, U, true, KEPT, 512>), grid, wg, 0, st, a);
        else if (p.r == 2) hipLaunchKernelGGL((qblock_norm_bwd_kernel<T, 2, U, true, KEPT, 256>), grid, wg, 0, st, a);
        else hipLaunchKernelGGL((qblock_norm_bwd_kernel<T, 8, U, true, KEPT, 256>), grid, wg, 0, st, a);
    } else {
        hipLaunchKernelGGL((qblock_norm_bwd_kernel<T, 2, U, false, KEPT, kThreads>), grid, wg, 0, st, a);
        if (a.out) {
            launch_norm_join<false>(a, st);
            hipLaunchKernelGGL((qblock_norm_dx_kernel<T, U, KEPT>), grid, wg, 0, st, a);
        }
    }
}

template <typename T, int U> void launch_norm_bwd_kept(const NormPlan &p, const NormArgs &a, bool kept, hipStream_t st) {
    if (kept) launch_norm_bwd_unit<T, U, true>(p, a, st);
    else launch_norm_bwd_unit<T, U, false>(p, a, st);
}

template <typename T> void launch_norm_bwd_of(const NormPlan &p, const NormArgs &a, bool kept, hipStream_t st) {
    if (p.u == 8) launch_norm_bwd_kept<T, 8>(p, a, kept, st);
    else if (p.u == 4) launch_norm_bwd_kept<T, 4>(p, a, kept, st);
    else if (p.u == 2) launch_norm_bwd_kept<T, 2>(p, a, kept, st);
    else launch_norm_bwd_kept<T, 1>(p, a, kept, st);
}

}  // namespace host
}  // namespace ql
