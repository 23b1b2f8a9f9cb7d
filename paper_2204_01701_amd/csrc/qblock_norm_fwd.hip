// qblock_norm_fwd.hip -- launches of the group normalization's forward.
#include "qblock_norm_host.h"

namespace ql {
namespace host {

namespace {

template <typename T, int U> void launch(const NormPlan &p, const NormArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)a.blocks), wg((unsigned)p.th);
    if (p.fused) {
        if (p.r > 8) {
            // (bf16's plan has none: 16 pixels a thread and two workgroups a CU do not fit the registers)
            if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((qblock_norm_fwd_kernel<T, 16, U, true, 512>), grid, wg, 0, st, a);
        } else if (p.th == 512) hipLaunchKernelGGL((qblock_norm_fwd_kernel<T, 8, U, true, 512>), grid, wg, 0, st, a);
        else if (p.r == 2) hipLaunchKernelGGL((qblock_norm_fwd_kernel<T, 2, U, true, 256>), grid, wg, 0, st, a);
        else hipLaunchKernelGGL((qblock_norm_fwd_kernel<T, 8, U, true, 256>), grid, wg, 0, st, a);
    } else {
        if (p.r == 2) hipLaunchKernelGGL((qblock_norm_fwd_kernel<T, 2, U, false, kThreads>), grid, wg, 0, st, a);
        else hipLaunchKernelGGL((qblock_norm_fwd_kernel<T, 8, U, false, kThreads>), grid, wg, 0, st, a);
        launch_norm_join<true>(a, st);
        hipLaunchKernelGGL((qblock_norm_apply_kernel<T, U>), grid, wg, 0, st, a);
    }
}

template <typename T> void launch_by_unit(const NormPlan &p, const NormArgs &a, hipStream_t st) {
    if (p.u == 8) launch<T, 8>(p, a, st);
    else if (p.u == 4) launch<T, 4>(p, a, st);
    else if (p.u == 2) launch<T, 2>(p, a, st);
    else launch<T, 1>(p, a, st);
}

}  // namespace

ql_status launch_norm_fwd(ql_dtype t, const NormPlan &p, const NormArgs &a, hipStream_t st) {
    if (t == QL_BF16) launch_by_unit<uint16_t>(p, a, st);
    else launch_by_unit<float>(p, a, st);
    return hip_status();
}

}  // namespace host
}  // namespace ql
