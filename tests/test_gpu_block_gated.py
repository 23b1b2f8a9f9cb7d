"""The gated layer against float64 definitions with elementwise bounds: every activation and tile, both types, one row to several
tiles, odd sizes, strides and alignments, checkpoints of both factors."""
import math

import pytest
import torch

import block_ref as ref
import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import gated_linear
from test_gpu_block_keep import DEV, TYPES, guarded, rows_of, type_ids

pytestmark = pytest.mark.gpu
ACTS = list(ql.HEAD_ACTS)


def inputs(m, k, n, dtype, seed=0):
    g = torch.Generator().manual_seed(m * 7919 + k * 31 + n + seed)
    x = torch.randn(m, k, generator=g).to(dtype)
    wg, wu = ((torch.randn(n, k, generator=g) / math.sqrt(k)).to(dtype) for _ in range(2))
    bg, bu = torch.randn(n, generator=g), torch.randn(n, generator=g)
    return x, wg, wu, bg, bu, torch.randn(m, n, generator=g).to(dtype), torch.randn(2, m, n, generator=g).to(dtype)


def forward(m, k, n, dtype, act="silu", bias=True, save=True, keep=False, offset=0, pad=0):
    x, wg, wu, bg, bu, _, _ = inputs(m, k, n, dtype)
    bg, bu = (bg, bu) if bias else (None, None)
    wide = torch.full((m, offset + n + pad), 77.0, device=DEV, dtype=dtype)
    h = wide[:, offset:offset + n]
    z, okz = guarded((2, m, n), dtype) if save else (None, lambda: True)
    q, okq = guarded((2, m, n), torch.int8) if keep else (None, lambda: True)
    e, oke = guarded((2, m, -(-n // 32)), torch.uint8) if keep else (None, lambda: True)
    ql.qblock_gated_fwd(rows_of(x, offset, pad), rows_of(wg, offset, pad), rows_of(wu, offset, pad),
                        *(b.to(DEV) if b is not None else None for b in (bg, bu)), h, z, q, e, act=act)
    want = ref.gated(x, wg, wu, bg, bu, act)
    ref.near(h, *want["h"], dtype)
    assert bool((wide[:, :offset] == 77).all() and (wide[:, offset + n:] == 77).all())
    for i, name in enumerate("gu"):
        v, ev = want[name]
        if save:
            ref.near(z[i], v, ev, dtype)
        if keep and m:
            got = ref.unpack(q[i].cpu(), e[i].cpu())
            blocks = torch.nn.functional.pad(v.abs() + ev, (0, -n % 32)).view(m, -1, 32).amax(2)
            # half a step, of at most 2 / 127 of the block's largest
            assert ((got - v).abs() <= (blocks / 127).repeat_interleave(32, 1)[:, :n] + ev).all()
            assert (torch.exp2(e[i].cpu().double() - 127) * 127 >= blocks * (1 - 2.0**-20) - ev.amax()).all()
    assert okz() and okq() and oke(), "written outside an output"


def backward(m, k, n, dtype, act="silu", keep=False, need=("dx", "dwg", "dwu", "dbg", "dbu"), offset=0, pad=0, wdtype=None):
    x, wg, wu, _, _, dh, z = inputs(m, k, n, dtype, 1)
    out = {"dx": guarded((m, k), dtype), "dwg": guarded((n, k), wdtype or dtype), "dwu": guarded((n, k), wdtype or dtype),
           "dbg": guarded((n,), torch.float32), "dbu": guarded((n,), torch.float32)}
    given = dict(z=z.to(DEV))
    if keep:
        q, e, z8 = ref.pack(z.view(2 * m, n))
        given = dict(q=q.to(DEV).view(2, m, n), e=e.to(DEV).view(2, m, -(-n // 32)))
        z = z8.view(2, m, n)
    ql.qblock_gated_bwd(rows_of(x, offset, pad), rows_of(wg, offset, pad), rows_of(wu, offset, pad), rows_of(dh, offset, pad), act=act,
                        **{name: out[name][0] if name in need else None for name in out}, **given)
    want = ref.gated_grads(x, wg, wu, dh, z[0], z[1], act, dtype)
    for name, (t, ok) in out.items():
        if name in need:
            ref.near(t, *want[name], t.dtype)
        else:
            assert bool((t == 77).all())
        assert ok(), "written outside an output"


# rows, inputs, outputs: single ones, a vector and its neighbours, K steps and tiles and theirs, long reductions
SIZES = [(1, 1, 1), (1, 8, 1), (2, 7, 3), (1, 64, 10), (3, 100, 17), (5, 33, 64), (16, 128, 130), (17, 256, 65), (64, 512, 10),
         (65, 64, 63), (128, 96, 256), (200, 72, 129), (257, 520, 300), (1, 4096, 70), (4, 1000, 1000), (40, 2048, 31), (300, 40, 600)]


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, dtype):
    forward(m, k, n, dtype)
    forward(m, k, n, dtype, "none", bias=False, save=False, offset=8, pad=8)
    forward(m, k, n, dtype, "gelu", save=False, keep=True, offset=1, pad=2)
    forward(m, k, n, dtype, "relu", bias=False, keep=True)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("m,k,n", SIZES)
def test_backward(m, k, n, dtype):
    backward(m, k, n, dtype)
    backward(m, k, n, dtype, "none", offset=8, pad=8)
    backward(m, k, n, dtype, "gelu", keep=True, offset=1, pad=2)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, dtype):
    forward(70, 72, 80, dtype, act)
    forward(9, 72, 80, dtype, act)
    backward(70, 72, 80, dtype, act)
    backward(70, 72, 80, dtype, act, keep=True)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
def test_only_what_is_asked_for(dtype):
    for need in (("dx",), ("dwg", "dwu"), ("dbg",), ("dbu",), ("dx", "dbg", "dbu")):
        backward(100, 40, 24, dtype, "gelu", need=need)
        backward(33, 41, 24, dtype, "gelu", need=need, keep=True)
    x, wg, wu, _, _, dh, z = (t.to(DEV) for t in inputs(20, 24, 40, dtype))
    dx = torch.empty(20, 24, device=DEV, dtype=dtype)
    ql.qblock_gated_bwd(None, wg, wu, dh, z, dx)
    ref.near(dx, *ref.gated_grads(x.cpu(), wg.cpu(), wu.cpu(), dh.cpu(), *z.cpu(), "silu", dtype)["dx"], dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("m,k,n", [(600, 1024, 768), (1030, 520, 520), (2100, 264, 128), (48, 3000, 512), (1, 3000, 5000), (33, 512, 4100)])
def test_larger(m, k, n, dtype):
    forward(m, k, n, dtype, "gelu_tanh")
    backward(m, k, n, dtype, "silu", keep=m < 100)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("tile,splits", [(0, 1), (0, 3), (1, 1), (1, 2), (2, 1), (2, 2)])
@pytest.mark.parametrize("m,k,n", [(300, 200, 264), (520, 1040, 128), (70, 96, 1031)])
def test_every_tile(m, k, n, tile, splits, dtype, monkeypatch):
    """Each tile on the same product, whatever the size would choose."""
    monkeypatch.setenv("QBLOCK_TILE", str(tile))
    monkeypatch.setenv("QBLOCK_SPLITS", str(splits))
    forward(m, k, n, dtype, "silu", keep=True, offset=8, pad=8)
    for both in range(2):  # the backward's products in turn, or in one launch
        monkeypatch.setenv("QBLOCK_BOTH", str(both))
        backward(m, k, n, dtype, "gelu", offset=1, pad=4)
        backward(m, k, n, dtype, "gelu", need=("dx",) if splits > 1 else ("dwg", "dwu"))


def test_float32_weight_gradients():
    backward(130, 72, 80, torch.bfloat16, "silu", wdtype=torch.float32)
    backward(130, 71, 80, torch.bfloat16, "silu", wdtype=torch.float32, keep=True)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
def test_no_rows(dtype):
    forward(0, 9, 5, dtype)
    backward(0, 9, 5, dtype)
    backward(0, 16, 40, dtype, keep=True)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("m", [3, 130])
def test_special_values_stay_in_their_rows(m, dtype):
    x, wg, wu, bg, bu, dh, z = inputs(m, 40, 72, dtype)
    x[1, 3], x[2, 0] = math.nan, math.inf
    h = torch.empty(m, 72, device=DEV, dtype=dtype)
    ql.qblock_gated_fwd(x.to(DEV), wg.to(DEV), wu.to(DEV), bg.to(DEV), bu.to(DEV), h, act="none")
    got = h.cpu()
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[2]).any()
    keep = [i for i in range(m) if i not in (1, 2)]
    ref.near(got[keep], *ref.gated(x[keep], wg, wu, bg, bu, "none")["h"], dtype)
    # a block of the checkpoint with a NaN: that row's gradients, and no other row's
    q, e, _ = ref.pack(z.view(2 * m, 72))
    e[1, 2] = 255
    dx = torch.empty(m, 40, device=DEV, dtype=dtype)
    ql.qblock_gated_bwd(None, wg.to(DEV), wu.to(DEV), dh.to(DEV), dx=dx, q=q.to(DEV).view(2, m, 72), e=e.to(DEV).view(2, m, 3))
    assert torch.isnan(dx[1]).all() and torch.isfinite(dx[[0] + list(range(2, m))]).all()


def test_same_results_every_time():
    x, wg, wu, bg, bu, dh, z = (t.to(DEV) for t in inputs(300, 520, 700, torch.bfloat16))
    outs = []
    for _ in range(3):
        h, zz = torch.empty_like(dh), torch.empty_like(z)
        ql.qblock_gated_fwd(x, wg, wu, bg, bu, h, zz)
        dx, dwg, dwu, dbg, dbu = (torch.empty_like(t) for t in (x, wg, wu, bg, bu))
        ql.qblock_gated_bwd(x, wg, wu, dh, z, dx, dwg, dwu, dbg, dbu)
        outs.append((h, zz, dx, dwg, dwu, dbg, dbu))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))


@pytest.mark.parametrize("act", [a for a in ACTS if a != "relu"])
def test_autograd_against_differences(act):
    """fp32 gradients of every leaf along random directions against central differences in float64."""
    g = torch.Generator().manual_seed(11)
    x, wg, wu, bg, bu, dh, _ = inputs(15, 24, 18, torch.float32, 2)
    x, dh = x.view(3, 5, 24), dh.view(3, 5, 18)
    leaves = [t.to(DEV).requires_grad_(True) for t in (x, wg, wu, bg, bu)]
    h = gated_linear(*leaves, act=act)
    assert h.shape == (3, 5, 18)
    grads = torch.autograd.grad(h, leaves, dh.to(DEV))

    def f(x, wg, wu, bg, bu):
        return (dh.double() * ref.act(x @ wg.t() + bg, act) * (x @ wu.t() + bu)).sum().item()

    at, step = [t.double() for t in (x, wg, wu, bg, bu)], 1e-6
    for i, grad in enumerate(grads):
        assert grad.shape == at[i].shape
        v = torch.randn(at[i].shape, generator=g, dtype=torch.float64)
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + step * v, at[i] - step * v
        got, scale = (grad.double().cpu() * v).sum().item(), (grad.double().cpu().abs() * v.abs()).sum().item()
        assert abs(got - (f(*up) - f(*down)) / (2 * step)) <= 2e-6 * scale + 1e-7 * dh.abs().sum().item()


def test_autograd_layouts():
    """Transposed inputs, halves of one weight, weights of another dtype, gradients that nobody asked for."""
    x = torch.randn(20, 6, device=DEV).t().requires_grad_(True)
    w = torch.randn(18, 20, device=DEV, requires_grad=True)
    h = gated_linear(x, w[:9], w[9:])
    gx, gw = torch.autograd.grad(h.sum(), (x, w))
    xd, wd = x.detach().double().cpu().requires_grad_(True), w.detach().double().cpu().requires_grad_(True)
    rx, rw = torch.autograd.grad((torch.nn.functional.silu(xd @ wd[:9].t()) * (xd @ wd[9:].t())).sum(), (xd, wd))
    assert torch.allclose(gx.double().cpu(), rx, atol=1e-3, rtol=1e-5) and torch.allclose(gw.double().cpu(), rw, atol=1e-3, rtol=1e-5)
    wb = torch.randn(9, 20, device=DEV, dtype=torch.bfloat16, requires_grad=True)
    h = gated_linear(x.detach(), wb, w[9:].detach()[:, :20])
    g, = torch.autograd.grad(h.sum(), wb)
    assert g.dtype == torch.bfloat16 and g.shape == wb.shape
    with torch.no_grad():
        assert not gated_linear(x, w[:9], w[9:], checkpoint="int8").requires_grad
    assert gated_linear(torch.empty(2, 0, 20, device=DEV), w[:9], w[9:]).shape == (2, 0, 9)


WRONG = [lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 9), t(6, 9), None, None, t(4, 6)), lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8), t(7, 8), None, None, t(4, 6)),
         lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8), t(6, 16)[:, :8], None, None, t(4, 6)), lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8), t(6, 8), t(5), None, t(4, 6)),
         lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8), t(6, 8), None, None, t(4, 7)), lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8), t(6, 8), None, None, t(4, 6), t(4, 12)),
         lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8).bfloat16(), t(6, 8), None, None, t(4, 6)), lambda t: ql.qblock_gated_fwd(t(8, 4).t(), t(6, 8), t(6, 8), None, None, t(4, 6)),
         lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8), t(6, 8), None, None, t(4, 6), q=t(2, 4, 6).to(torch.int8)),
         lambda t: ql.qblock_gated_fwd(t(4, 8), t(6, 8), t(6, 8), None, None, t(4, 6), act="tanh"),
         lambda t: ql.qblock_gated_bwd(t(4, 8), t(6, 8), t(6, 8), t(4, 6), None, t(4, 8)), lambda t: ql.qblock_gated_bwd(t(4, 8), t(6, 8), t(6, 8), t(4, 6), t(2, 4, 6), dwg=t(6, 8)),
         lambda t: ql.qblock_gated_bwd(None, t(6, 8), t(6, 8), t(4, 6), t(2, 4, 6), dwg=t(6, 8), dwu=t(6, 8)),
         lambda t: ql.qblock_gated_bwd(t(4, 8), t(6, 8), t(6, 8), t(4, 6), t(2, 4, 6), dwg=t(6, 8), dwu=t(6, 8).bfloat16()),
         lambda t: ql.qblock_gated_bwd(t(5, 8), t(6, 8), t(6, 8), t(4, 6), t(2, 4, 6), t(4, 8)),
         lambda t: gated_linear(t(4, 8), t(6, 9), t(6, 9)), lambda t: gated_linear(t(4, 8), t(6, 8), t(7, 8)), lambda t: gated_linear(t(4, 8), t(6, 8), t(6, 8), t(5)),
         lambda t: gated_linear(t(4, 8), t(6, 8), torch.zeros(6, 8))]


@pytest.mark.parametrize("k", range(len(WRONG)))
def test_wrong_tensors(k):
    with pytest.raises(ValueError):
        WRONG[k](lambda *s: torch.zeros(*s, device=DEV))


def test_nothing_asked_for():
    t = torch.zeros(4, 8, device=DEV)
    with pytest.raises(ql.QLError):
        ql.qblock_gated_bwd(t, t, t, torch.zeros(4, 4, device=DEV), torch.zeros(2, 4, 4, device=DEV))
