"""Host-side checks of the operators at the end of a network that need no GPU: the exported
symbols, the refusals of the C ABI (before anything is launched), workspace queries, and
the binding's refusals of tensors that are not on a GPU."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2204_01701_amd as ql
from paper_2204_01701_amd import build as qbuild
from paper_2204_01701_amd.autograd import distill_loss, linear_act, token_logprobs

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qhead.h")
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
P = 0x10000  # stands for a device pointer: refused calls never look behind it
BF, F = ql.QL_BF16, ql.QL_F32


@pytest.fixture(scope="module")
def L():
    if qbuild.is_stale():
        qbuild.build()
    return ql.lib()


def test_exports_and_header(L, tmp_path):
    txt = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(qhead_\w+)\s*\(", txt)))
    assert len(names) == 11
    out = subprocess.run(["nm", "-D", "--defined-only", ql.LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = set(re.findall(r"\bT (qhead_\w+)", out))
    assert exported == set(names)
    src = tmp_path / "h.c"
    src.write_text('#include "qhead.h"\nint main(void) { return QL_ACT_SILU + QHEAD_MAX_TOP == 132 ? 0 : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), "-c", str(src), "-o", str(tmp_path / "h.o")],
                   check=True)
    assert f"QHEAD_MAX_TOP {ql.HEAD_MAX_TOP}" in open(HEADER).read()


def lin(m=4, k=8, n=6, ldx=None, ldw=None, ldr=None, ldy=None, dtype=BF, act=0):
    return ctypes.byref(ql.HeadLinearDesc(m, k, n, k if ldx is None else ldx, k if ldw is None else ldw,
                                          n if ldr is None else ldr, n if ldy is None else ldy, dtype, act))


BIG = 1 << 40


@pytest.mark.parametrize("bad", [dict(m=-1), dict(k=0), dict(n=0), dict(k=-3), dict(ldx=7), dict(ldw=7), dict(ldy=5), dict(ldr=5),
                                 dict(dtype=2), dict(act=5), dict(act=-1)])
def test_linear_refuses_descriptors(L, bad):
    assert L.qhead_linear_fwd(lin(**bad), P, P, P, P, P, None, P, BIG, None) == EINVAL
    if "ldr" not in bad:
        assert L.qhead_linear_bwd(lin(**bad), P, P, P, P, P, P, P, P, BIG, None) == EINVAL


def test_linear_refuses_sizes_at_the_end_of_int(L):
    for big in (dict(m=2**31 - 2), dict(k=2**31 - 2), dict(n=2**31 - 2)):
        assert L.qhead_linear_fwd(lin(**big), P, P, P, P, P, None, P, BIG, None) == EUNSUPPORTED
        assert L.qhead_linear_bwd(lin(**big), P, P, P, P, P, P, P, P, BIG, None) == EUNSUPPORTED


def test_linear_refuses_pointers(L):
    for i in (0, 1, 4):  # x, w, y
        args = [P, P, P, P, P, None]
        args[i] = None
        assert L.qhead_linear_fwd(lin(), *args, P, BIG, None) == EINVAL
        args[i] = P + 1
        assert L.qhead_linear_fwd(lin(), *args, P, BIG, None) == EINVAL
    assert L.qhead_linear_fwd(lin(dtype=F), P + 2, P, P, P, P, None, P, BIG, None) == EINVAL
    assert L.qhead_linear_fwd(lin(), P, P, P + 2, P, P, None, P, BIG, None) == EINVAL
    assert L.qhead_linear_bwd(lin(), P, P, P, P, None, None, None, P, BIG, None) == EINVAL  # nothing asked for
    assert L.qhead_linear_bwd(lin(act=2), P, P, P, None, P, None, None, P, BIG, None) == EINVAL  # an activation without z
    assert L.qhead_linear_bwd(lin(), P, None, P, None, P, None, None, P, BIG, None) == EINVAL
    assert L.qhead_linear_bwd(lin(), None, P, P, None, None, P, None, P, BIG, None) == EINVAL
    assert L.qhead_linear_bwd(lin(), P, P, None, None, P, None, None, P, BIG, None) == EINVAL
    need = L.qhead_linear_bwd_workspace_size(lin(act=2))
    assert need > 0
    assert L.qhead_linear_bwd(lin(act=2), P, P, P, P, P, P, P, None, 0, None) == EWORKSPACE
    assert L.qhead_linear_bwd(lin(act=2), P, P, P, P, P, P, P, P, need - 1, None) == EWORKSPACE
    assert L.qhead_linear_bwd(lin(act=2), P, P, P, P, P, P, P, P + 8, need, None) == EINVAL
    assert L.qhead_linear_fwd(lin(m=0), None, None, None, None, None, None, None, 0, None) == OK


def rows(r=4, v=50, ld=None, top=3, dtype=BF, t=1.0, alpha=1.0):
    return ctypes.byref(ql.HeadRowsDesc(r, v, v if ld is None else ld, top, dtype, t, alpha))


BAD = [dict(r=-1), dict(v=0), dict(ld=49), dict(dtype=7), dict(t=0.0), dict(t=-1.0), dict(t=float("nan")), dict(t=float("inf")),
       dict(top=-1), dict(top=129)]


@pytest.mark.parametrize("bad", BAD + [dict(v=2)])
def test_logprobs_refuses_descriptors(L, bad):
    assert L.qhead_logprobs_fwd(rows(**bad), P, P, P, P, P, P, P, P, P, BIG, None) == EINVAL
    if "top" not in bad and bad != dict(v=2):
        assert L.qhead_logprobs_bwd(rows(**bad), P, P, P, P, P, P, P + 64, None) == EINVAL


@pytest.mark.parametrize("bad", BAD + [dict(alpha=-0.1), dict(alpha=1.1), dict(alpha=float("nan"))])
def test_distill_refuses_descriptors(L, bad):
    assert L.qhead_distill_fwd(rows(**bad), P, P, P, P, P, P, P, BIG, None) == EINVAL
    assert L.qhead_distill_bwd(rows(**bad), P, P, P, P, P, P, P + 64, None) == EINVAL
    assert L.qhead_distill_step(rows(**bad), P, P, P, P, P, P, P + 64, P, BIG, None) == EINVAL


def test_rows_refuse_pointers(L):
    def without(f, desc, args, i, tail):
        for v in (None, args[i] + 1):
            a = list(args)
            a[i] = v
            assert f(desc, *a, *tail) == EINVAL, (f.__name__, i, v)

    for i in (0, 1, 2, 5, 6):
        without(L.qhead_logprobs_fwd, rows(), [P] * 8, i, (P, BIG, None))
    for i in (0, 1, 2, 3, 4, 6):  # the entropy belongs to h
        without(L.qhead_logprobs_bwd, rows(), [P] * 6 + [P + 64], i, (None,))
    for i in (0, 1, 2, 4):
        without(L.qhead_distill_fwd, rows(), [P] * 6, i, (P, BIG, None))
    for i in (0, 1, 2, 4, 5, 6):
        without(L.qhead_distill_bwd, rows(), [P] * 6 + [P + 64], i, (None,))
        without(L.qhead_distill_step, rows(), [P] * 6 + [P + 64], i, (P, BIG, None))
    # in place only where the rows lie side by side
    assert L.qhead_distill_step(rows(ld=64), P, P, P, P, P, P, P, P, BIG, None) == EINVAL
    assert L.qhead_logprobs_bwd(rows(ld=64), P, P, P, P, P, P, P, None) == EINVAL
    # few long rows are split over workgroups and need a workspace
    for size, call, args in ((L.qhead_logprobs_fwd_workspace_size, L.qhead_logprobs_fwd, [P] * 8),
                             (L.qhead_distill_workspace_size, L.qhead_distill_step, [P] * 6 + [P + 64])):
        need = size(rows(v=200000))
        assert need > 0 and size(rows()) == 0
        assert call(rows(v=200000), *args, None, 0, None) == EWORKSPACE
        assert call(rows(v=200000), *args, P, need - 1, None) == EWORKSPACE
    assert L.qhead_logprobs_fwd(rows(r=0), *[None] * 8, None, 0, None) == OK
    assert L.qhead_distill_step(rows(r=0), *[None] * 7, None, 0, None) == OK


def test_binding_refuses_cpu_tensors():
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    with pytest.raises(ValueError):
        ql.qhead_linear_fwd(x, w, None, None, torch.zeros(4, 6))
    with pytest.raises(ValueError):
        ql.qhead_logprobs_fwd(x, torch.zeros(4, dtype=torch.int64), torch.zeros(4))
    with pytest.raises(ValueError):
        ql.qhead_distill_fwd(x, None, None, None, torch.zeros(4))
    with pytest.raises(ValueError):
        linear_act(x, w)
    with pytest.raises(ValueError):
        token_logprobs(x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        distill_loss(x, None, None, torch.zeros(4, dtype=torch.int64))
