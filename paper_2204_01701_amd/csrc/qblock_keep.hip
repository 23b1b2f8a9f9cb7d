// qblock_keep.hip -- host side of the 8-bit checkpoints of include/qblock.h.
#include "qblock_host.h"

using namespace ql;
using namespace ql::host;

namespace ql {
namespace host {

ql_status run_keep(bool pack, ql_dtype t, void *x, long long ld, int8_t *q, uint8_t *e, long long rows, long long cols, hipStream_t st) {
    if (rows == 0) return QL_OK;
    if (ld == cols && cols % kKeep == 0) {  // one long row
        cols *= rows;
        ld = cols;
        rows = 1;
    }
    const KeepArgs a{x, ld, q, e, rows, cols, (cols + kKeep - 1) / kKeep};
    const dim3 grid((unsigned)std::min<long long>((a.rows * a.blocks * 4 + kThreads - 1) / kThreads, 1 << 20)), wg(kThreads);
    if (pack && t == QL_BF16) hipLaunchKernelGGL((qblock_pack8_kernel<uint16_t>), grid, wg, 0, st, a);
    else if (pack) hipLaunchKernelGGL((qblock_pack8_kernel<float>), grid, wg, 0, st, a);
    else if (t == QL_BF16) hipLaunchKernelGGL((qblock_unpack8_kernel<uint16_t>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((qblock_unpack8_kernel<float>), grid, wg, 0, st, a);
    return hip_status();
}

}  // namespace host
}  // namespace ql

namespace {

ql_status keep(bool pack, const qblock_keep_desc *d, void *x, int8_t *q, uint8_t *e, void *stream) {
    if (!d || d->rows < 0 || d->cols < 1 || d->ld < d->cols || !float_type(d->dtype)) return QL_EINVAL;
    if (d->cols > kMostInt || d->rows > (1LL << 47) / d->cols || d->ld > (1LL << 47)) return QL_EUNSUPPORTED;
    if (d->rows == 0) return QL_OK;
    if (!x || !q || !e || !aligned(x, esize(d->dtype))) return QL_EINVAL;
    return run_keep(pack, d->dtype, x, d->rows > 1 ? d->ld : d->cols, q, e, d->rows, d->cols, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

ql_status qblock_pack8(const qblock_keep_desc *d, const void *x, int8_t *q, uint8_t *e, void *stream) {
    return keep(true, d, const_cast<void *>(x), q, e, stream);
}

ql_status qblock_unpack8(const qblock_keep_desc *d, const int8_t *q, const uint8_t *e, void *x, void *stream) {
    return keep(false, d, x, const_cast<int8_t *>(q), const_cast<uint8_t *>(e), stream);
}

}  // extern "C"
