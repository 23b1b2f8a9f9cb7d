// qblock_norm_bwd_bf16.hip -- launches of the group normalization's backward, bf16.
#include "qblock_norm_bwd.h"

namespace ql {
namespace host {

template void launch_norm_bwd_of<uint16_t>(const NormPlan &p, const NormArgs &a, bool kept, hipStream_t st);

}  // namespace host
}  // namespace ql
