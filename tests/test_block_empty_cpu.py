"""Batches of no rows at the C ABI, whose tensors may be NULL as those of an empty torch tensor are: nothing to do is no error."""
import ctypes
import os
import re

import pytest

import paper_2204_01701_amd as ql
from paper_2204_01701_amd import build as qbuild

OK, EINVAL = 0, 1
P = 0x10000  # stands for a device pointer: no call here launches anything


@pytest.fixture(scope="module")
def L():
    if qbuild.is_stale():
        qbuild.build()
    return ql.lib()


@pytest.mark.parametrize("dtype", [ql.QL_BF16, ql.QL_F32], ids=["bf16", "fp32"])
def test_norm_gradient_of_the_map_alone(L, dtype):
    def desc(n):
        return ctypes.byref(ql.BlockNormDesc(n, 9, 12, 3, dtype, 4, 1.0))
    assert L.qblock_norm_bwd(desc(0), *[None] * 11, None, 0, None) == OK
    assert L.qblock_norm_bwd(desc(0), P, None, P, P, None, None, P, P, P, None, None, None, 0, None) == OK
    assert L.qblock_norm_bwd(desc(1), *[P] * 8, None, None, None, P, 1 << 60, None) == EINVAL


@pytest.mark.parametrize("dtype", [ql.QL_BF16, ql.QL_F32], ids=["bf16", "fp32"])
def test_gated_gradient_of_the_input_alone(L, dtype):
    def desc(m):
        return ctypes.byref(ql.BlockGatedDesc(m, 16, 24, 16, 16, 24, dtype, 4, 0, 0))
    assert L.qblock_gated_bwd(desc(0), *[None] * 12, None, 0, None) == OK
    assert L.qblock_gated_bwd(desc(0), P, P, P, P, P, None, None, P, None, None, None, None, None, 0, None) == OK
    assert L.qblock_gated_bwd(desc(1), *[P] * 5, None, None, *[None] * 5, P, 1 << 60, None) == EINVAL


@pytest.mark.parametrize("dtype", [ql.QL_BF16, ql.QL_F32], ids=["bf16", "fp32"])
def test_first_order_gradient_of_the_input_alone(L, dtype):
    def desc(m):
        return ctypes.byref(ql.HeadLinearDesc(m, 16, 24, 16, 16, 24, 24, dtype, 4, 0, 0))
    assert L.qhead_linear_bwd(desc(0), *[None] * 7, None, 0, None) == OK
    assert L.qhead_linear_bwd(desc(0), P, P, P, P, P, None, None, None, 0, None) == OK
    assert L.qhead_linear_bwd(desc(1), P, P, P, P, None, None, None, P, 1 << 60, None) == EINVAL


def test_constants_of_the_header():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qblock.h")).read()
    assert dict(re.findall(r"#define (QBLOCK_\w+) (\d+)", header)) == {"QBLOCK_KEEP": str(ql.BLOCK_KEEP), "QBLOCK_FEW_ROWS": str(ql.BLOCK_FEW_ROWS)}
