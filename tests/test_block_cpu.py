"""Host-side checks of the operators of include/qblock.h that need no GPU: exported symbols, refusals of the C ABI
(before anything is launched), workspace queries, the binding's refusals, the checkpoint's definition."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import block_ref as ref
import paper_2204_01701_amd as ql
from paper_2204_01701_amd import autograd as ag
from paper_2204_01701_amd import build as qbuild

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qblock.h")
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
P = 0x10000  # stands for a device pointer: refused calls never look behind it
BF, F = ql.QL_BF16, ql.QL_F32
BIG = 1 << 60


@pytest.fixture(scope="module")
def L():
    if qbuild.is_stale():
        qbuild.build()
    return ql.lib()


def test_exports_and_header(L, tmp_path):
    txt = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(qblock_\w+)\s*\(", txt)))
    assert len(names) == 10
    out = subprocess.run(["nm", "-D", "--defined-only", ql.LIB_PATH], capture_output=True, text=True, check=True).stdout
    assert set(re.findall(r"\bT (qblock_\w+)", out)) == set(names)
    src = tmp_path / "h.c"
    src.write_text('#include "qblock.h"\nint main(void) { qblock_gated_desc d; qblock_norm_desc n; qblock_keep_desc k;\n'
                   f'return sizeof d == {ctypes.sizeof(ql.BlockGatedDesc)} && sizeof n == {ctypes.sizeof(ql.BlockNormDesc)} && '
                   f'sizeof k == {ctypes.sizeof(ql.BlockKeepDesc)} && QBLOCK_KEEP == {ql.BLOCK_KEEP} ? 0 : 1; }}\n')
    exe = str(tmp_path / "h")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), "-o", exe, str(src)], check=True)
    assert subprocess.run([exe]).returncode == 0


# --- checkpoints ---------------------------------------------------------------------

def keep(rows=4, cols=40, ld=None, dtype=BF):
    return ctypes.byref(ql.BlockKeepDesc(rows, cols, cols if ld is None else ld, dtype))


@pytest.mark.parametrize("bad,want", [(dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(ld=39), EINVAL), (dict(dtype=2), EINVAL),
                                      (dict(cols=2**31 - 2, ld=2**31), EUNSUPPORTED), (dict(rows=1 << 46), EUNSUPPORTED)])
def test_checkpoints_refuse(L, bad, want):
    assert L.qblock_pack8(keep(**bad), P, P, P, None) == want
    assert L.qblock_unpack8(keep(**bad), P, P, P, None) == want


def test_checkpoints_refuse_pointers(L):
    for i in range(3):
        args = [P, P, P]
        args[i] = None
        assert L.qblock_pack8(keep(), *args, None) == EINVAL
        assert L.qblock_unpack8(keep(), *args, None) == EINVAL
    assert L.qblock_pack8(keep(), P + 1, P, P, None) == EINVAL
    assert L.qblock_unpack8(keep(dtype=F), P, P, P + 2, None) == EINVAL
    assert L.qblock_pack8(None, P, P, P, None) == EINVAL
    assert L.qblock_pack8(keep(rows=0), None, None, None, None) == OK


def test_the_checkpoints_definition():
    """The reference itself: least exponents, halves to even, the error bound, blocks without a value."""
    x = torch.tensor([[127.0, 126.5, 125.5, -0.5, 1.5], [127.5, 1.0, 3.0, -3.0, 0.0], [0.0] * 5, [1.0, math.nan, 0, 0, 0]])
    q, e, x8 = ref.pack(x)
    assert e[:, 0].tolist() == [127, 128, 1, 255]
    assert q[0].tolist() == [127, 126, 126, 0, 2] and q[1].tolist() == [64, 0, 2, -2, 0]
    assert torch.isnan(x8[3]).all() and torch.equal(ref.unpack(q, e)[:3], x8[:3])
    g = torch.Generator().manual_seed(0)
    y = torch.randn(50, 70, generator=g) * torch.exp2(torch.randint(-100, 100, (50, 1), generator=g).float())
    q, e, y8 = ref.pack(y)
    for b in range(3):
        part = y[:, 32 * b:32 * b + 32].double()
        assert ((part - y8[:, 32 * b:32 * b + 32]).abs() <= part.abs().amax(1, keepdim=True) / 127).all()
    assert torch.equal(y8.to(torch.bfloat16).double(), y8) and int(q.abs().max()) <= 127


# --- group norm ----------------------------------------------------------------------

def norm(n=2, hw=9, c=12, groups=3, dtype=BF, act=1, eps=1e-5):
    return ctypes.byref(ql.BlockNormDesc(n, hw, c, groups, dtype, act, eps))


def norm_calls(L, d, eps_matters=True):
    yield L.qblock_norm_fwd(d, P, P, P, P, P, P, P, P, P, BIG, None)
    if not eps_matters:
        yield L.qblock_norm_bwd(d, P, P, None, None, P, P, P, P, P, P, P, P, BIG, None)


@pytest.mark.parametrize("bad,want", [(dict(n=-1), EINVAL), (dict(hw=0), EINVAL), (dict(c=0), EINVAL), (dict(groups=0), EINVAL),
                                      (dict(groups=5), EINVAL), (dict(dtype=7), EINVAL), (dict(act=5), EINVAL), (dict(act=-1), EINVAL),
                                      (dict(n=2**31 - 2), EUNSUPPORTED), (dict(hw=2**31 - 2), EUNSUPPORTED),
                                      (dict(c=(1 << 20) + 2), EUNSUPPORTED),
                                      (dict(n=2**30, hw=2**20), EUNSUPPORTED)])
def test_norm_refuses_descriptors(L, bad, want):
    for status in norm_calls(L, norm(**bad), False):
        assert status == want


@pytest.mark.parametrize("eps", [0.0, -1e-5, math.inf, math.nan])
def test_norm_refuses_eps(L, eps):
    for status in norm_calls(L, norm(eps=eps)):
        assert status == EINVAL


def test_norm_refuses_pointers(L):
    for i, off in ((0, None), (3, None), (0, 1), (3, 1), (1, 2), (2, 2), (4, 2), (5, 2), (6, None), (7, None)):
        args = [P] * 8
        args[i] = None if off is None else P + off
        assert L.qblock_norm_fwd(norm(), *args, P, BIG, None) == EINVAL, i
    for i, off in ((0, None), (6, None), (7, None), (0, 1), (1, 1), (8, 1), (4, 2), (5, 2), (6, 2), (7, 2), (9, 2), (10, 2)):
        args = [P] * 11
        args[i] = None if off is None else P + off
        assert L.qblock_norm_bwd(norm(), *args, P, BIG, None) == EINVAL, i
    full = [P] * 11
    assert L.qblock_norm_bwd(norm(), *full[:8], None, None, None, P, BIG, None) == EINVAL  # nothing asked for
    assert L.qblock_norm_bwd(norm(), P, None, P, None, *full[4:], P, BIG, None) == EINVAL  # half a checkpoint
    assert L.qblock_norm_bwd(norm(), P, None, None, None, *full[4:], P, BIG, None) == EINVAL
    assert L.qblock_norm_fwd(norm(n=0), *[None] * 8, None, 0, None) == OK


def test_norm_workspaces(L):
    for d in (norm(), norm(n=4, hw=10000, c=64, groups=8), norm(n=1, hw=1, c=1 << 20, groups=1), norm(n=1, hw=5, c=6000, groups=2)):
        for query, call, args in ((L.qblock_norm_fwd_workspace_size, L.qblock_norm_fwd, [P] * 8),
                                  (L.qblock_norm_bwd_workspace_size, L.qblock_norm_bwd, [P] * 11)):
            need = query(d)
            if need:
                assert call(d, *args, P, need - 1, None) == EWORKSPACE
                assert call(d, *args, None, need, None) == EWORKSPACE
                assert call(d, *args, P + 8, need, None) == EINVAL
    assert L.qblock_norm_bwd_workspace_size(norm()) > 0
    assert L.qblock_norm_fwd_workspace_size(norm(n=4, hw=10000, c=64, groups=8)) > 0
    assert L.qblock_norm_fwd_workspace_size(norm(c=-4)) == 0 and L.qblock_norm_bwd_workspace_size(norm(n=0)) == 0


# --- gated layer -----------------------------------------------------------------------

def gated(m=40, k=16, n=24, ldx=None, ldw=None, ldh=None, dtype=BF, act=4, unaligned=0, dw_f32=0):
    return ctypes.byref(ql.BlockGatedDesc(m, k, n, k if ldx is None else ldx, k if ldw is None else ldw, n if ldh is None else ldh,
                                          dtype, act, unaligned, dw_f32))


@pytest.mark.parametrize("bad,want", [(dict(m=-1), EINVAL), (dict(k=0), EINVAL), (dict(n=0), EINVAL), (dict(ldx=15), EINVAL),
                                      (dict(ldw=15), EINVAL), (dict(ldh=23), EINVAL), (dict(dtype=3), EINVAL), (dict(act=9), EINVAL),
                                      (dict(m=2**31 - 2), EUNSUPPORTED), (dict(k=(1 << 19) + 8), EUNSUPPORTED),
                                      (dict(n=(1 << 19) + 8), EUNSUPPORTED)])
def test_gated_refuses_descriptors(L, bad, want):
    assert L.qblock_gated_fwd(gated(**bad), *[P] * 9, P, BIG, None) == want
    assert L.qblock_gated_bwd(gated(**bad), *[P] * 12, P, BIG, None) == want


def test_gated_refuses_pointers(L):
    for i, off in ((0, None), (1, None), (2, None), (5, None), (7, None), (8, None), (0, 1), (5, 1), (6, 1), (3, 2), (4, 2)):
        args = [P] * 9
        args[i] = None if off is None else P + off
        assert L.qblock_gated_fwd(gated(), *args, P, BIG, None) == EINVAL, i
    for i, off in ((0, None), (1, None), (2, None), (3, None), (8, None), (9, None), (0, 1), (3, 1), (4, 1), (7, 1), (8, 1), (10, 2), (11, 2)):
        args = [P] * 12
        args[i] = None if off is None else P + off
        assert L.qblock_gated_bwd(gated(), *args, P, BIG, None) == EINVAL, i
    a = [P] * 12
    assert L.qblock_gated_bwd(gated(), *a[:7], None, None, None, None, None, P, BIG, None) == EINVAL  # nothing asked for
    assert L.qblock_gated_bwd(gated(), *a[:4], None, P, None, *a[7:], P, BIG, None) == EINVAL  # half a checkpoint
    assert L.qblock_gated_bwd(gated(dw_f32=1), *a[:8], P + 2, *a[9:], P, BIG, None) == EINVAL
    # 2 bytes off: refused unless announced (then the workspace holds copies), or few rows that are read in place
    for i in range(3):
        args = [P] * 9
        args[i] = P + 2
        assert L.qblock_gated_fwd(gated(), *args, P, BIG, None) == EINVAL
        assert L.qblock_gated_fwd(gated(unaligned=1), *args, None, 0, None) == EWORKSPACE
        args = [P] * 12
        args[i] = P + 2
        assert L.qblock_gated_bwd(gated(), *args, P, BIG, None) == EINVAL
    assert L.qblock_gated_fwd(gated(m=0), *[None] * 9, None, 0, None) == OK


def test_gated_workspaces(L):
    for d in (gated(k=17), gated(ldx=19), gated(m=500, n=500, k=4000), gated(dtype=F, k=18)):
        for query, call, args in ((L.qblock_gated_fwd_workspace_size, L.qblock_gated_fwd, [P] * 9),
                                  (L.qblock_gated_bwd_workspace_size, L.qblock_gated_bwd, [P] * 12)):
            need = query(d)
            if need:
                assert call(d, *args, P, need - 1, None) == EWORKSPACE
                assert call(d, *args, P + 8, need, None) == EINVAL
        assert L.qblock_gated_bwd_workspace_size(d) > 0
    assert L.qblock_gated_fwd_workspace_size(gated()) == 0
    assert L.qblock_gated_fwd_workspace_size(gated(k=17)) < L.qblock_gated_fwd_workspace_size(gated(k=17, m=400))


# --- the binding and the autograd functions, without a GPU ------------------------------

CPU = [lambda t: ql.qblock_pack8(t(4, 40), t(4, 40), t(4, 2)), lambda t: ql.qblock_unpack8(t(4, 40), t(4, 2), t(4, 40)),
       lambda t: ql.qblock_norm_fwd(t(2, 9, 12), 3, None, None, t(2, 9, 12)),
       lambda t: ql.qblock_norm_bwd(t(2, 9, 12), t(2, 9, 12), 3, None, None, t(2, 3), t(2, 3), t(2, 9, 12)),
       lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8), t(6, 8), None, None, t(4, 6)),
       lambda t: ql.qblock_gated_bwd(t(4, 8), t(6, 8), t(6, 8), t(4, 6), t(2, 4, 6), t(4, 8)),
       lambda t: ag.group_norm_act(t(2, 12, 3, 3), 3), lambda t: ag.gated_linear(t(4, 8), t(6, 8), t(6, 8))]


@pytest.mark.parametrize("i", range(len(CPU)))
def test_tensors_on_the_cpu_are_refused(i):
    with pytest.raises(ValueError):
        CPU[i](torch.zeros)


@pytest.mark.parametrize("call", [lambda x, w, k: ag.quad_linear(x, w, w, w, checkpoint=k), lambda x, w, k: ag.linear_act(x, w, checkpoint=k),
                                  lambda x, w, k: ag.gated_linear(x, w, w, checkpoint=k), lambda x, w, k: ag.group_norm_act(x, 2, checkpoint=k),
                                  lambda x, w, k: ag.quad_conv2d(x, w, checkpoint=k)])
def test_unknown_checkpoints_are_refused(call):
    with pytest.raises(ValueError, match="checkpoint"):
        call(torch.zeros(4, 8), torch.zeros(6, 8), "fp8")


@pytest.fixture
def calls(monkeypatch):
    """The library's calls replaced by stand-ins that compute nothing; each call's name and pointers."""
    seen = []
    monkeypatch.setattr(ag, "_same_device", lambda *tensors: None)
    monkeypatch.setattr(ag, "_block_launch", lambda name, desc, ptrs, index, query=None: seen.append((name, ptrs)))
    for name in ("qhead_linear_fwd", "qhead_linear_bwd"):
        monkeypatch.setattr(ag, name, lambda *args, _name=name, **kw: seen.append((_name, args)))
    return seen


def layers(checkpoint):
    def leaf(*s):
        return torch.randn(*s, requires_grad=True)
    return {"norm": ((leaf(2, 12, 3, 3), leaf(12), leaf(12)), lambda x, w, b: ag.group_norm_act(x, 3, w, b, act="silu", checkpoint=checkpoint)),
            "rows": ((leaf(5, 12), leaf(12), leaf(12)), lambda x, w, b: ag.group_norm_act(x, 3, w, b, checkpoint=checkpoint)),
            "gated": ((leaf(2, 3, 5), leaf(4, 5), leaf(4, 5), leaf(4), leaf(4)), lambda *a: ag.gated_linear(*a, checkpoint=checkpoint)),
            "linear": ((leaf(3, 5), leaf(4, 5), leaf(4)), lambda *a: ag.linear_act(*a, act="gelu", checkpoint=checkpoint))}


@pytest.mark.parametrize("checkpoint", [None, "int8"])
@pytest.mark.parametrize("which", ["norm", "rows", "gated", "linear"])
def test_gradients_arrive_and_a_second_derivative_raises(calls, which, checkpoint):
    """In 8 bits, where nothing ties a gradient to the activation, already a backward that a second one could follow."""
    leaves, f = layers(checkpoint)[which]
    y = f(*leaves)
    grads = torch.autograd.grad(y.sum(), leaves, retain_graph=True)
    for leaf, g in zip(leaves, grads):
        assert g.shape == leaf.shape and not g.requires_grad
    for i in range(len(leaves) if which != "linear" else 2):
        with pytest.raises(RuntimeError, match="twice"):
            g, = torch.autograd.grad(y.sum(), leaves[i], create_graph=True, retain_graph=True)
            torch.autograd.grad(g.square().sum(), leaves[0], retain_graph=True, allow_unused=True)


@pytest.mark.parametrize("which", ["norm", "gated", "linear"])
def test_what_a_checkpoint_keeps(calls, which):
    """In 8 bits: nothing of the forward's dtype but the parameters and statistics is kept, and x is not either."""
    leaves, f = layers("int8")[which]
    y = f(*leaves)
    kept = [t for t in y.grad_fn.saved_tensors if t is not None]
    for t in kept:
        assert t.dtype in (torch.int8, torch.uint8) or any(t.shape == leaf.shape for leaf in leaves[1:]) or t.shape == (2, 2, 3)
    assert leaves[0].data_ptr() not in {t.data_ptr() for t in kept}


@pytest.mark.parametrize("off", [torch.no_grad, torch.inference_mode])
def test_serving_writes_nothing_for_a_backward(calls, off):
    with off():
        for which in ("norm", "gated", "linear"):
            leaves, f = layers("int8")[which]
            assert not f(*leaves).requires_grad
    assert [name for name, _ in calls] == ["qblock_norm_fwd", "qblock_gated_fwd", "qhead_linear_fwd"]
    assert calls[0][1][4:] == (None,) * 4  # mean, rstd, q, e
    assert calls[1][1][6:] == (None,) * 3 and calls[2][1][5] is None  # z, q, e; z


def test_only_what_is_asked_for(calls):
    (x, wg, wu, bg, bu), f = layers("int8")["gated"]
    y = f(x, wg.detach(), wu.detach(), bg, bu)
    y.sum().backward()
    assert [name for name, _ in calls] == ["qblock_gated_fwd", "qblock_gated_bwd"]  # (x is not packed: no weight needs it)
    px, *_, dx, dwg, dwu, dbg, dbu = calls[1][1]
    assert px is None and dwg is None and dwu is None and dx and dbg and dbu and x.grad is not None and wg.grad is None
