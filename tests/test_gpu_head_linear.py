"""The first-order layer (product, bias, activation, residual; its gradients) against float64
definitions with elementwise bounds: every activation, both types, sizes from one row, one
input and one output to several tiles, row strides and alignments, special values, refusals of
nothing that the sizes allow."""
import math

import pytest
import torch

import head_ref as ref
import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import linear_act

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float32]
type_ids = ["bf16", "fp32"]
ACTS = list(ql.HEAD_ACTS)


def _gen(*key):
    return torch.Generator().manual_seed(hash(tuple(key)) % (1 << 31))


def _rows(t, offset, pad, foreign=math.nan):
    """t on the GPU as rows of a wider tensor, `offset` elements from its start, foreign values around."""
    r, c = t.shape
    wide = torch.full((r, offset + c + pad), foreign, dtype=t.dtype)
    wide[:, offset:offset + c] = t
    return wide.to(DEV)[:, offset:offset + c]


def _guarded(shape, dtype):
    n = math.prod(shape)
    raw = torch.full((n + 128,), 77, dtype=dtype, device=DEV)
    return raw[64:64 + n].view(shape), lambda: bool((raw[:64] == 77).all() and (raw[64 + n:] == 77).all())


def _inputs(m, k, n, dtype, seed=0):
    g = _gen(m, k, n, seed)
    x = torch.randn(m, k, generator=g).to(dtype)
    w = (torch.randn(n, k, generator=g) / math.sqrt(k)).to(dtype)
    b = torch.randn(n, generator=g)
    r, dy = torch.randn(m, n, generator=g).to(dtype), torch.randn(m, n, generator=g).to(dtype)
    return x, w, b, r, dy


def _fwd(m, k, n, dtype, act, bias=True, res=True, save=True, offset=0, pad=0, xs=None):
    x, w, b, r, _ = _inputs(m, k, n, dtype)
    if xs is not None:
        x = xs
    b, r = b if bias else None, r if res else None
    y, ok = _guarded((m, n), dtype)
    z, okz = _guarded((m, n), dtype)
    ql.qhead_linear_fwd(_rows(x, offset, pad), _rows(w, offset, pad), b.to(DEV) if bias else None,
                        _rows(r, offset, pad) if res else None, y, z if save else None, act=act)
    ry, rz, ey, ez = ref.linear(x, w, b, r, act)
    ref.near(y, ry, ey, dtype)
    if save:
        ref.near(z, rz, ez, dtype)
    assert ok() and okz(), "written outside an output"


def _bwd(m, k, n, dtype, act, need=("dx", "dw", "db"), offset=0, pad=0):
    x, w, _, z, dy = _inputs(m, k, n, dtype, 1)
    out = {"dx": _guarded((m, k), dtype), "dw": _guarded((n, k), dtype), "db": _guarded((n,), torch.float32)}
    give = {name: out[name][0] if name in need else None for name in out}
    ql.qhead_linear_bwd(_rows(x, offset, pad), _rows(w, offset, pad), _rows(dy, offset, pad),
                        z.to(DEV) if act != "none" else None, **give, act=act)
    want = ref.linear_grads(x, w, dy, z, act)
    for name, (t, ok) in out.items():
        if name in need:
            ref.near(t, *want[name], t.dtype)
        else:
            assert bool((t == 77).all())
        assert ok(), "written outside an output"


# rows, inputs, outputs: single ones, a vector and its neighbours, a tile and its neighbours, several tiles, long reductions
SIZES = [(1, 1, 1), (1, 8, 1), (2, 7, 3), (1, 64, 10), (3, 100, 17), (5, 33, 64), (16, 128, 130), (17, 257, 65), (64, 512, 10),
         (65, 64, 63), (128, 96, 256), (200, 72, 129), (257, 513, 300), (1, 4096, 70), (4, 1000, 1000), (40, 2049, 31),
         (300, 40, 600), (520, 256, 264)]


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, dtype):
    _fwd(m, k, n, dtype, "gelu")
    _fwd(m, k, n, dtype, "none", bias=False, res=False, save=False, offset=8, pad=8)
    _fwd(m, k, n, dtype, "silu", res=False, offset=1, pad=2)
    _fwd(m, k, n, dtype, "relu", bias=False, save=False, offset=3)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("m,k,n", SIZES)
def test_backward(m, k, n, dtype):
    _bwd(m, k, n, dtype, "gelu")
    _bwd(m, k, n, dtype, "none", offset=8, pad=8)
    _bwd(m, k, n, dtype, "silu", offset=1, pad=2)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, dtype):
    _fwd(70, 72, 80, dtype, act)
    _bwd(70, 72, 80, dtype, act)
    for need in (("dx",), ("dw",), ("db",), ("dx", "db")):
        _bwd(33, 40, 24, dtype, act, need)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("m,k,n", [(600, 1024, 768), (1030, 520, 520), (2100, 264, 128), (48, 3000, 512), (1, 3000, 5000), (33, 512, 4100)])
def test_larger(m, k, n, dtype):
    _fwd(m, k, n, dtype, "gelu_tanh")
    _bwd(m, k, n, dtype, "relu")


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("tile,splits", [(128, 1), (128, 3), (256, 1), (256, 2), (64, 1), (64, 2), (1, 1)])
@pytest.mark.parametrize("m,k,n", [(300, 200, 264), (520, 1040, 128), (70, 96, 1031)])
def test_every_tile(m, k, n, tile, splits, dtype, monkeypatch):
    """Each tile on the same product, whatever the size would choose."""
    monkeypatch.setenv("QHEAD_TILE", str(tile))
    monkeypatch.setenv("QHEAD_SPLITS", str(splits))
    _fwd(m, k, n, dtype, "silu", offset=8, pad=8)
    _bwd(m, k, n, dtype, "gelu", offset=1, pad=4)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
def test_no_rows(dtype):
    _fwd(0, 9, 5, dtype, "gelu")
    _bwd(0, 9, 5, dtype, "gelu")


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("m,k,n", [(3, 40, 20), (130, 264, 136)])
def test_special_values_stay_in_their_rows(m, k, n, dtype):
    """NaN and infinities of a row of x reach that row's outputs and no others; large activations saturate."""
    x = _inputs(m, k, n, dtype)[0]
    x[1, 3], x[2, 0] = math.nan, math.inf
    w, b, r = (v for v in _inputs(m, k, n, dtype)[1:4])
    y = torch.empty(m, n, device=DEV, dtype=dtype)
    ql.qhead_linear_fwd(x.to(DEV), w.to(DEV), b.to(DEV), r.to(DEV), y, act="none")
    got = y.cpu()
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[2]).any()
    keep = [i for i in range(m) if i not in (1, 2)]
    ry, _, ey, _ = ref.linear(x[keep], w, b, r[keep], "none")
    ref.near(got[keep], ry, ey, dtype)
    for act in ("relu", "gelu", "gelu_tanh", "silu"):
        big = torch.tensor([[1e4], [-1e4], [1e30], [-1e30], [0.0], [-0.0]]).to(dtype)
        one = torch.ones(1, 1, dtype=dtype)
        out, z, dx = (torch.empty(6, 1, device=DEV, dtype=dtype) for _ in range(3))
        ql.qhead_linear_fwd(big.to(DEV), one.to(DEV), None, None, out, z, act=act)
        ref.near(out, big.double().clamp_min(0), torch.full((6, 1), 1e-30, dtype=torch.float64), dtype)
        ql.qhead_linear_bwd(big.to(DEV), one.to(DEV), torch.ones(6, 1, dtype=dtype, device=DEV), z, dx, act=act)
        slope = (big > 0).double()
        if act != "relu":
            slope[4:] = 0.5
        ref.near(dx, slope, torch.full((6, 1), 1e-30, dtype=torch.float64), dtype)


def test_residual_may_be_the_output():
    x, w, b, r, _ = _inputs(130, 72, 80, torch.bfloat16)
    y = r.to(DEV)
    ql.qhead_linear_fwd(x.to(DEV), w.to(DEV), b.to(DEV), y, y, act="silu")
    ry, _, ey, _ = ref.linear(x, w, b, r, "silu")
    ref.near(y, ry, ey, torch.bfloat16)


@pytest.mark.parametrize("act", ACTS)
def test_autograd_against_differences(act):
    """fp32 gradients of x, w, b and the residual along random directions against central differences in float64
    (z stays off relu's kink by the inputs' seed at the step used)."""
    g = _gen(21)
    x, w, b, r, dy = (v.view(3, 5, -1) if i in (0, 3, 4) else v for i, v in enumerate(_inputs(15, 24, 18, torch.float32, 2)))
    leaves = [v.to(DEV).requires_grad_(True) for v in (x, w, b, r)]
    y = linear_act(*leaves, act=act)
    assert y.shape == (3, 5, 18)
    grads = torch.autograd.grad(y, leaves, dy.to(DEV))

    def f(*v):
        return (dy.double() * (ref.act(v[0] @ v[1].t() + v[2], act) + v[3])).sum().item()

    at, h = [v.double() for v in (x, w, b, r)], 1e-6
    for i, grad in enumerate(grads):
        assert grad.shape == at[i].shape
        v = torch.randn(at[i].shape, generator=g, dtype=torch.float64)
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * v, at[i] - h * v
        got, scale = (grad.double().cpu() * v).sum().item(), (grad.double().cpu().abs() * v.abs()).sum().item()
        assert abs(got - (f(*up) - f(*down)) / (2 * h)) <= 2e-6 * scale


def test_autograd_layouts():
    """Transposed and expanded inputs, weights of another dtype, gradients that nobody asked for."""
    x = torch.randn(20, 6, device=DEV).t().requires_grad_(True)
    w = torch.randn(9, 20, device=DEV, dtype=torch.bfloat16).requires_grad_(True)
    y = linear_act(x, w, torch.ones(9, device=DEV), torch.ones(1, device=DEV).expand(6, 9), act="relu")
    y.sum().backward()  # an expanded upstream gradient
    ref_y = torch.relu(x.detach().double() @ w.detach().double().t() + 1) + 1
    assert torch.allclose(y.double(), ref_y, atol=1e-4)
    mask = (ref_y > 1).double()
    assert torch.allclose(x.grad.double(), mask @ w.detach().double(), atol=1e-4)
    assert w.grad.dtype == torch.bfloat16
    assert torch.allclose(w.grad.double(), mask.t().contiguous() @ x.detach().double(), atol=0.05)
    with torch.no_grad():
        assert not linear_act(x, w).requires_grad
    assert linear_act(torch.empty(2, 0, 20, device=DEV), w).shape == (2, 0, 9)
