// qblock_host.h -- what the host sides of include/qblock.h share.
#pragma once

#include "qblock.h"
#include "qblock_keep.h"
#include "qhost.h"

namespace ql {
namespace host {

constexpr int kMostInt = 0x7fffffff - 65536;  // (the kernels' counters run past a size by up to a few thousand)

inline size_t esize(ql_dtype t) { return t == QL_BF16 ? 2 : 4; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool float_type(ql_dtype t) { return t == QL_F32 || t == QL_BF16; }
inline bool known_act(ql_act a) { return (int)a >= QL_ACT_NONE && (int)a <= QL_ACT_SILU; }

// x -> q, e (pack) or back; arguments are checked.
ql_status run_keep(bool pack, ql_dtype t, void *x, long long ld, int8_t *q, uint8_t *e, long long rows, long long cols, hipStream_t st);

}  // namespace host
}  // namespace ql
