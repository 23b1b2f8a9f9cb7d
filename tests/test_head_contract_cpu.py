"""What include/qhead.h states of its arguments, held against the entry points without a GPU:
every call here is refused before anything is launched, or has no rows."""
import ctypes

import pytest

import paper_2204_01701_amd as ql
from paper_2204_01701_amd import build as qbuild

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
P = 0x10000  # stands for a device pointer: refused calls never look behind it
BF, F = ql.QL_BF16, ql.QL_F32
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    if qbuild.is_stale():
        qbuild.build()
    return ql.lib()


def rows(r=4, v=50, ld=None, top=3, dtype=BF, t=1.0, alpha=0.5, f32=0):
    return ctypes.byref(ql.HeadRowsDesc(r, v, v if ld is None else ld, top, dtype, t, alpha, f32))


def test_a_float32_teacher_is_aligned_to_four_bytes(L):
    # (a workspace too small ends the calls whose arguments are in order)
    for f32, dtype, off, want in ((0, BF, 2, EWORKSPACE), (1, BF, 2, EINVAL), (1, BF, 4, EWORKSPACE), (0, F, 2, EINVAL)):
        d = rows(v=200000, dtype=dtype, f32=f32)
        assert L.qhead_distill_fwd(d, P, P, P + off, P, P, P, None, 0, None) == want
        assert L.qhead_distill_step(d, P, P, P + off, P, P, P, P + 64, None, 0, None) == want
    assert L.qhead_distill_bwd(rows(f32=1), P, P, P + 2, P, P, P, P + 64, None) == EINVAL


def test_a_float32_weight_gradient_is_aligned_to_four_bytes(L):
    def lin(dw_f32):
        return ctypes.byref(ql.HeadLinearDesc(4, 8, 6, 8, 8, 6, 6, BF, ql.HEAD_ACTS["gelu"], 0, dw_f32))

    for f32, off, want in ((0, 2, EWORKSPACE), (1, 2, EINVAL), (1, 4, EWORKSPACE)):
        assert L.qhead_linear_bwd(lin(f32), P, P, P, P, P, P + off, P, None, 0, None) == want


def test_the_distillations_statistics_are_aligned_to_their_elements(L):
    # (a workspace too small, or g misaligned, ends the calls whose stats are in order)
    for off, want in ((4, EWORKSPACE), (8, EWORKSPACE), (2, EINVAL)):
        assert L.qhead_distill_fwd(rows(v=200000), P, P, P, P, P, P + off, None, 0, None) == want
    assert L.qhead_distill_bwd(rows(), P, P, P, P, P + 2, P, P + 64, None) == EINVAL


@pytest.mark.parametrize("t,scores,distils", [(4.2e-39, False, False), (1e-44, False, False), (4.3e-39, True, True), (1e-30, True, True),
                                              (1.8e19, True, True), (1.9e19, True, False), (3e38, True, False)])
def test_temperatures_that_float32_cannot_carry_are_refused(L, t, scores, distils):
    d, want = rows(v=200000, t=t), {True: EWORKSPACE, False: EINVAL}
    assert L.qhead_logprobs_fwd(d, P, P, P, P, P, P, P, P, None, 0, None) == want[scores]
    assert L.qhead_distill_fwd(d, P, P, P, P, P, P, None, 0, None) == want[distils]
    assert L.qhead_distill_step(d, P, P, P, P, P, P, P + 64, None, 0, None) == want[distils]
    if not scores:
        assert L.qhead_logprobs_bwd(d, P, P, P, P, P, P, P + 64, None) == EINVAL
    if not distils:
        assert L.qhead_distill_bwd(d, P, P, P, P, P, P, P + 64, None) == EINVAL
