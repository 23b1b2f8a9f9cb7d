"""The first-order layer's weight gradient in float32 beside bfloat16 operands, and the bfloat16
gradients of linear_act, against float64."""
import pytest
import torch

import head_ref as ref
import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import linear_act

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def _inputs(m, k, n, seed):
    g = torch.Generator().manual_seed(seed)
    x, dy = torch.randn(m, k, generator=g).to(BF), torch.randn(m, n, generator=g).to(BF)
    w = torch.randn(n, k, generator=g) / k ** 0.5
    return x, w, dy, torch.randn(m, n, generator=g).to(BF), torch.randn(n, generator=g)


# one row and one element, element by element, each tile, splits with their join, copies of odd layouts, no rows
@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (5, 7, 3), (64, 512, 10), (257, 513, 300), (300, 200, 264), (2100, 264, 128),
                                   (4096, 256, 256), (600, 1024, 768), (0, 9, 5)])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_float32_weight_gradient(m, k, n, act):
    x, w, dy, z, _ = _inputs(m, k, n, 51)
    raw = torch.full((n * k + 128,), 77.0, device=DEV)
    dw, dx, db = raw[64:64 + n * k].view(n, k), torch.empty(m, k, device=DEV, dtype=BF), torch.empty(n, device=DEV)
    ql.qhead_linear_bwd(x.to(DEV), w.to(BF).to(DEV), dy.to(DEV), z.to(DEV), dx, dw, db, act=act)
    want = ref.linear_grads(x, w.to(BF), dy, z, act)
    ref.near(dw, *want["dw"], torch.float32)
    ref.near(dx, *want["dx"], BF)
    ref.near(db, *want["db"], torch.float32)
    assert bool((raw[:64] == 77).all() and (raw[64 + n * k:] == 77).all()), "written outside the gradient"
    half = torch.empty(n, k, device=DEV, dtype=BF)
    ql.qhead_linear_bwd(x.to(DEV), w.to(BF).to(DEV), dy.to(DEV), z.to(DEV), dw=half, act=act)
    assert torch.equal(half, dw.to(BF)), "the same sums, rounded once"


@pytest.mark.parametrize("tile,splits", [(128, 1), (128, 3), (256, 2), (64, 1), (1, 1)])
def test_every_tile(tile, splits, monkeypatch):
    monkeypatch.setenv("QHEAD_TILE", str(tile))
    monkeypatch.setenv("QHEAD_SPLITS", str(splits))
    test_float32_weight_gradient(520, 264, 136, "silu")


def test_misfits_are_refused():
    x, w, dy = (torch.zeros(s, device=DEV, dtype=BF) for s in ((4, 8), (6, 8), (4, 6)))
    for bad in (torch.zeros(6, 9, device=DEV), torch.zeros(6, 8, device=DEV, dtype=torch.float16)):
        with pytest.raises(ValueError):
            ql.qhead_linear_bwd(x, w, dy, dw=bad)


@pytest.mark.parametrize("act", list(ql.HEAD_ACTS))
@pytest.mark.parametrize("wdtype", [BF, torch.float32])
def test_linear_act_in_bfloat16(act, wdtype):
    """Against the definitions at the pre-activation that the layer keeps, z rounded to bfloat16."""
    m, k, n = 130, 72, 200
    x, w, dy, r, b = _inputs(m, k, n, 52)
    w = w.to(wdtype)
    leaves = [v.to(DEV).requires_grad_(True) for v in (x, w, b, r)]
    y = linear_act(*leaves, act=act)
    ry, _, ey, _ = ref.linear(x, w.to(BF), b, r, act)
    ref.near(y, ry, ey, BF)
    z = torch.empty(m, n, device=DEV, dtype=BF)
    ql.qhead_linear_fwd(leaves[0].detach(), leaves[1].detach().to(BF), leaves[2].detach(), None, torch.empty_like(z), z, act=act)
    gx, gw, gb, gr = torch.autograd.grad(y, leaves, dy.to(DEV))
    want = ref.linear_grads(x, w.to(BF), dy, z.cpu(), act)
    ref.near(gx, *want["dx"], BF)
    assert gw.dtype is wdtype
    ref.near(gw, *want["dw"], wdtype)
    ref.near(gb, *want["db"], torch.float32)
    assert torch.equal(gr.cpu(), dy)
