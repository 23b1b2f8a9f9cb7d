// qblock_norm_bwd_f32.hip -- launches of the group normalization's backward, float32.
#include "qblock_norm_bwd.h"

namespace ql {
namespace host {

template void launch_norm_bwd_of<float>(const NormPlan &p, const NormArgs &a, bool kept, hipStream_t st);

}  // namespace host
}  // namespace ql
