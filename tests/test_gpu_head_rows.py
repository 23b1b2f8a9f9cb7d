"""The rows-of-logits operators (log probabilities, distillation) against float64 definitions:
sizes from one value a row to long rows split over workgroups, rows at every alignment and with
foreign values behind them, masked, empty, equal, rising, infinite and NaN rows, both types."""
import math

import pytest
import torch

import head_ref as ref
import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import distill_loss, token_logprobs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = math.inf, math.nan
TYPES = [torch.bfloat16, torch.float32]
type_ids = ["bf16", "fp32"]


def _gen(*key):
    return torch.Generator().manual_seed(hash(tuple(key)) % (1 << 31))


def _logits(rows, vocab, dtype, seed):
    g = _gen(rows, vocab, seed)
    return (torch.randn(rows, vocab, generator=g) * 3).to(dtype)


def _special(vocab, dtype, seed=0):
    """Rows that a mask, a sort or an overflow can trip over."""
    low, big = torch.finfo(dtype).min, torch.finfo(dtype).max
    g = _gen(vocab, seed)
    base = (torch.randn(vocab, generator=g) * 3).to(dtype)
    half = base.clone()
    half[torch.rand(vocab, generator=g) < 0.5] = -INF
    lows = base.clone()
    lows[torch.rand(vocab, generator=g) < 0.5] = low
    only = torch.full((vocab,), -INF, dtype=dtype)
    only[vocab // 2] = 1.5
    wide = base.clone()
    wide[0], wide[-1] = low, big
    nan, pinf = base.clone(), base.clone()
    nan[vocab // 3] = NAN
    pinf[vocab // 3] = INF
    zeros = torch.zeros(vocab, dtype=dtype)
    zeros[::2] = -0.0
    steps = torch.arange(vocab).div(7, rounding_mode="floor").to(dtype)
    rows = [base, torch.full((vocab,), -INF, dtype=dtype), torch.full((vocab,), low, dtype=dtype), zeros, half, lows, only,
            torch.sort(base)[0], torch.sort(base, descending=True)[0], steps, wide, nan, pinf, torch.full((vocab,), NAN, dtype=dtype)]
    return torch.stack(rows)


def _place(z, offset, pad, foreign=NAN):
    """z on the GPU as rows cut out of a wider tensor, `offset` elements from an aligned start; foreign values around."""
    rows, vocab = z.shape
    wide = torch.full((rows, vocab + pad + offset), foreign, dtype=z.dtype)
    wide[:, offset:offset + vocab] = z
    return wide.to(DEV)[:, offset:offset + vocab]


def _guarded(shape, dtype):
    """A tensor inside a larger one full of a pattern, and the check that the pattern around it stands."""
    n = math.prod(shape)
    raw = torch.full((n + 128,), 77, dtype=dtype, device=DEV)
    return raw[64:64 + n].view(shape), lambda: bool((raw[:64] == 77).all() and (raw[64 + n:] == 77).all())


def _score(z, target, top, t):
    rows = z.shape[0]
    (f, ok0), (tl, ok1), (ti, ok2) = (_guarded((3, rows), torch.float32), _guarded((rows, top), torch.float32),
                                      _guarded((rows, top), torch.int64))
    stats, ok3 = _guarded((rows, 2), torch.float32)
    ql.qhead_logprobs_fwd(z, target.to(DEV), f[0], f[1], f[2], tl if top else None, ti if top else None, stats, temperature=t)
    torch.cuda.synchronize()
    assert ok0() and ok1() and ok2() and ok3(), "written outside an output"
    return f[0], f[1], f[2], tl, ti, stats


def _check_score(z, zd, target, top, t):
    logp, ent, lse, tl, ti, stats = _score(zd, target, top, t)
    rl, rh, rs, el, eh, es = ref.logprobs(z, target, t)
    ref.near(logp, rl, el, torch.float32)
    ref.near(ent, rh, eh, torch.float32)
    ref.near(lse, rs, es, torch.float32)
    if top:
        order = ref.rank(z)[:, :top]
        assert torch.equal(ti.cpu(), order), "alternatives in another order"
        full = ref.softmax_parts(z, t)[0].gather(1, order)
        full = torch.where(torch.isnan(rs)[:, None], torch.full_like(full, NAN), full)
        bound = es[:, None] + 8 * ref.U32 * full.abs().nan_to_num(0, 0, 0)
        ref.near(tl, full, bound, torch.float32)
    return ent, stats


SIZES = [(3, 1, 1), (5, 2, 2), (4, 7, 7), (6, 10, 3), (3, 63, 20), (2, 64, 64), (3, 257, 128), (2, 512, 40), (2, 513, 128), (3, 1000, 5),
         (2, 2049, 64), (2, 4099, 20), (1, 16384, 128), (2, 33001, 64), (1, 70001, 128), (600, 130, 4), (0, 50, 3),
         (3, 1600, 128), (3, 1040, 128), (2, 2040, 64), (2100, 600, 128), (2100, 700, 64), (2100, 3001, 64)]


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("rows,vocab,top", SIZES)
def test_logprobs(rows, vocab, top, dtype):
    z = _logits(rows, vocab, dtype, 1)
    g = _gen(rows, vocab, 2)
    target = torch.randint(-2, vocab + 1, (rows,), generator=g)
    for offset, pad, t in ((0, 0, 1.0), (1, 6, 0.7), (3, 0, 4.0)):
        _check_score(z, _place(z, offset, pad), target, top, t)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("vocab,top", [(5, 5), (40, 20), (300, 128), (3001, 64), (20000, 128), (20000, 0), (50021, 20)])
def test_logprobs_special_rows(vocab, top, dtype):
    z = _special(vocab, dtype)
    g = _gen(vocab, 5)
    target = torch.randint(0, vocab, (z.shape[0],), generator=g)
    _check_score(z, _place(z, 1, 3), target, top, 1.0)
    _check_score(z, _place(z, 0, 0), torch.full_like(target, -100), top, 0.9)
    many = z.repeat(40, 1)  # rows that are not split
    _check_score(many, many.to(DEV), target.repeat(40), top, 1.0)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("rows,vocab", [(3, 1), (4, 9), (3, 1001), (2, 20003), (1200, 37), (0, 8)])
@pytest.mark.parametrize("with_h", [False, True])
def test_logprobs_grad(rows, vocab, dtype, with_h):
    z = torch.cat([_logits(rows, vocab, dtype, 3), _special(vocab, dtype)]) if rows else _logits(0, vocab, dtype, 3)
    n = z.shape[0]
    g = _gen(n, vocab, 4)
    target = torch.randint(-1, vocab + 1, (n,), generator=g)
    up, h = torch.randn(n, generator=g), torch.randn(n, generator=g) if with_h else None
    up[:1] = 0
    for offset, t in ((0, 1.0), (1, 2.5)):
        zd = _place(z, offset, offset)
        _, ent, _, _, _, stats = _score(zd, target, 0, t)
        dz, ok = _guarded((n, vocab), dtype)
        ql.qhead_logprobs_bwd(zd, target.to(DEV), stats, ent, up.to(DEV), h.to(DEV) if with_h else None, dz, temperature=t)
        want, bound = ref.logprobs_grad(z, target, t, up, h)
        ref.near(dz, want, bound, dtype)
        assert ok()
    if n:  # in place
        zd = z.to(DEV)
        ql.qhead_logprobs_bwd(zd, target.to(DEV), stats, ent, up.to(DEV), h.to(DEV) if with_h else None, zd, temperature=t)
        ref.near(zd, want, bound, dtype)


def _teacher(rows, vocab, top, dtype, seed):
    """Places of a teacher: distinct ids, ids twice, empty places, places of probability 0, rows without any."""
    g = _gen(rows, vocab, top, seed)
    ids = torch.stack([torch.randperm(max(vocab, top), generator=g)[:top] % vocab for _ in range(rows)]) if rows else torch.zeros(0, top, dtype=torch.long)
    tz = (torch.randn(rows, top, generator=g) * 3).to(dtype)
    ids[torch.rand(rows, top, generator=g) < 0.1] = -1
    if top > 1:
        ids[::3, 1] = ids[::3, 0]
        tz[1::4, 0] = -INF
    if rows > 2:
        ids[2] = -5
    if rows > 3:
        tz[3] = -INF
    if rows > 4:
        tz[4] = torch.finfo(dtype).min
    return ids, tz


HOW = [(1.0, 1.0), (2.0, 1.0), (2.0, 0.4), (1.0, 0.4), (3.0, 0.0)]


def _check_distill(z, zd, ids, tz, label, up, t, alpha, tag=""):
    rows, vocab = z.shape
    dev = lambda v: v.to(DEV) if v is not None else None  # noqa: E731
    want, grad, el, eg = ref.distill(z, ids, tz, label, t, alpha, up)
    how = dict(temperature=t, alpha=alpha)
    (loss, ok0), (stats, ok1), (dz, ok2) = (_guarded((rows,), torch.float32), _guarded((rows, 4), torch.float32),
                                            _guarded((rows, vocab), z.dtype))
    ql.qhead_distill_fwd(zd, dev(ids), dev(tz), dev(label), loss, stats, **how)
    ref.near(loss, want, el, torch.float32)
    ql.qhead_distill_bwd(zd, dev(ids), dev(tz), dev(label), stats, dev(up), dz, **how)
    ref.near(dz, grad, eg, z.dtype)
    assert ok0() and ok1() and ok2()
    (loss, ok0), (dz, ok2) = _guarded((rows,), torch.float32), _guarded((rows, vocab), z.dtype)
    ql.qhead_distill_step(zd, dev(ids), dev(tz), dev(label), dev(up), loss, dz, **how)
    ref.near(loss, want, el, torch.float32)
    ref.near(dz, grad, eg, z.dtype)
    assert ok0() and ok2()
    if rows:
        over = z.to(DEV)
        ql.qhead_distill_step(over, dev(ids), dev(tz), dev(label), dev(up), loss, over, **how)
        ref.near(over, grad, eg, z.dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("rows,vocab,top", [(3, 1, 1), (7, 10, 10), (5, 33, 20), (6, 1001, 64), (5, 20003, 128), (300, 257, 31),
                                            (0, 20, 4), (4, 40, 0), (5, 3, 7)])
def test_distill(rows, vocab, top, dtype):
    z = _logits(rows, vocab, dtype, 6)
    g = _gen(rows, vocab, 7)
    ids, tz = _teacher(rows, vocab, top, dtype, 8)
    label = torch.randint(-1, vocab, (rows,), generator=g)
    if top and rows:
        label[0] = ids[0, 0].clamp_min(0)
    up = torch.randn(rows, generator=g)
    for i, (t, alpha) in enumerate(HOW):
        _check_distill(z, _place(z, i % 3, 2 * i), ids if top else None, tz if top else None, None if alpha == 1.0 and i else label,
                       up, t, alpha)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("vocab", [6, 700, 9001])
def test_distill_special_rows(vocab, dtype):
    z = _special(vocab, dtype, 3)
    rows = z.shape[0]
    ids, tz = _teacher(rows, vocab, 5, dtype, 9)
    ids[5, 2] = vocab  # past the vocabulary
    g = _gen(vocab, 10)
    label = torch.randint(-1, vocab, (rows,), generator=g)
    label[6] = vocab + 3
    up = torch.randn(rows, generator=g)
    up[-2] = 0  # a row that counts for nothing, +inf in it
    for t, alpha in HOW:
        _check_distill(z, _place(z, 1, 1), ids, tz, label, up, t, alpha)
        none = torch.full_like(ids, -1)  # no row has a term: nothing in a row may reach its gradient
        _check_distill(z, z.to(DEV), none, tz, torch.full_like(label, -1), up, t, alpha)


def _direction(z, v, f, h=1e-4):
    return (f(z + h * v) - f(z - h * v)) / (2 * h)


@pytest.mark.parametrize("vocab", [9, 1003])
def test_gradients_against_differences(vocab):
    """The fp32 gradients along random directions against central differences of the float64 definitions (step 1e-4:
    truncation ~ h^2 / 6 |f'''| < 1e-7 of the gradient's scale, rounding 1e-16 / h)."""
    rows = 6
    z = _logits(rows, vocab, torch.float32, 11)
    g = _gen(vocab, 12)
    target = torch.randint(0, vocab, (rows,), generator=g)
    up, h = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    ids, tz = _teacher(rows, vocab, min(5, vocab), torch.float32, 13)
    leaf = z.to(DEV).requires_grad_(True)
    logp, ent = token_logprobs(leaf, target.to(DEV), temperature=1.7)
    one, = torch.autograd.grad((logp, ent), leaf, (up.to(DEV), h.to(DEV)))
    two, = torch.autograd.grad(distill_loss(leaf, ids.to(DEV), tz.to(DEV), target.to(DEV), temperature=1.7, alpha=0.6), leaf, up.to(DEV))

    def f1(x):
        a = ref.logprobs(x, target, 1.7)
        return (up.double() * a[0] + h.double() * a[1]).sum()

    def f2(x):
        return (up.double() * ref.distill(x, ids, tz, target, 1.7, 0.6, up)[0]).sum()

    for k in range(4):
        v = torch.randn(rows, vocab, generator=g, dtype=torch.float64)
        for grad, f in ((one, f1), (two, f2)):
            got = (grad.double().cpu() * v).sum().item()
            scale = (grad.double().cpu().abs() * v.abs()).sum().item()
            assert abs(got - _direction(z.double(), v, f).item()) <= 1e-5 * scale + 1e-9


def test_autograd_shapes_and_partial_gradients():
    z = _logits(12, 50, torch.float32, 14).view(3, 4, 50).to(DEV).requires_grad_(True)
    target = torch.randint(0, 50, (3, 4), device=DEV)
    logp, ent, tl, ti = token_logprobs(z, target, top=5)
    assert logp.shape == ent.shape == (3, 4) and tl.shape == ti.shape == (3, 4, 5) and ti.dtype == torch.int64
    assert not tl.requires_grad and not ti.requires_grad
    want = torch.log_softmax(z.double(), -1)
    a, = torch.autograd.grad(ent.sum(), z, retain_graph=True)  # an expanded upstream gradient, none for logp
    b, = torch.autograd.grad(-(want.exp() * want).sum(), z, retain_graph=True)
    assert torch.allclose(a, b, atol=1e-6)
    a, = torch.autograd.grad(logp.mean(), z, retain_graph=True)
    again, = torch.autograd.grad(logp.mean(), z)
    assert torch.equal(a, again)
    b, = torch.autograd.grad(want.gather(-1, target[..., None]).mean(), z)
    assert torch.allclose(a, b, atol=1e-7)
    loss = distill_loss(z.transpose(0, 1), ti.transpose(0, 1), tl.transpose(0, 1), target.t(), temperature=2.0, alpha=0.5)
    assert loss.shape == (4, 3)
    loss.sum().backward()
    assert z.grad.shape == z.shape and torch.isfinite(z.grad).all()
    no_rows = token_logprobs(z[:0], target[:0], top=2)
    assert no_rows[0].shape == (0, 4) and no_rows[2].shape == (0, 4, 2)


def test_streams_and_repeats():
    """On another stream than the default one, repeated: the same bits."""
    z = _logits(5, 30011, torch.bfloat16, 15).to(DEV)
    target = torch.arange(5, device=DEV)
    first = _score(z, target, 33, 1.3)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        for _ in range(3):
            again = _score(z, target, 33, 1.3)
    st.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_graph_capture():
    """A captured step replays to the eager result, on new inputs too."""
    rows, vocab, top = 6, 20011, 16
    z = _logits(rows, vocab, torch.bfloat16, 16).to(DEV)
    target = torch.arange(rows, device=DEV)
    f = torch.zeros(2, rows, device=DEV)
    tl, ti = torch.zeros(rows, top, device=DEV), torch.zeros(rows, top, device=DEV, dtype=torch.int64)
    loss, up, dz = torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV), torch.zeros_like(z)

    def step():
        ql.qhead_logprobs_fwd(z, target, f[0], f[1], None, tl, ti)
        ql.qhead_distill_step(z, ti, tl.to(z.dtype), target, up, loss, dz, temperature=2.0, alpha=0.5)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step()
    torch.cuda.current_stream().wait_stream(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        z.copy_(_logits(rows, vocab, torch.bfloat16, 17 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (f, tl, ti, loss, dz)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (f, tl, ti, loss, dz)):
            assert torch.equal(a, b)


def test_long_offsets():
    """Rows whose offsets pass 2^32 elements."""
    vocab, ld = 70000, 1 << 30
    wide = torch.empty(5 * ld, dtype=torch.bfloat16, device=DEV)
    z = wide.view(5, ld)[:, 3:3 + vocab]
    host = _logits(5, vocab, torch.bfloat16, 18)
    z.copy_(host)
    target = torch.arange(5)
    _, _, _, tl, ti, _ = _score(z, target, 8, 1.0)
    _check_score(host, z, target, 8, 1.0)
    loss, dz = torch.empty(5, device=DEV), torch.empty(5, vocab, device=DEV, dtype=torch.bfloat16)
    ql.qhead_distill_step(z, ti, tl.bfloat16(), None, torch.ones(5, device=DEV), loss, dz, temperature=1.0)
    want, grad, el, eg = ref.distill(host, ti.cpu(), tl.bfloat16().cpu(), None, 1.0, 1.0, torch.ones(5))
    ref.near(loss, want, el, torch.float32)
    ref.near(dz, grad, eg, torch.bfloat16)


LONG = [(256, 2000, 20), (256, 9001, 128), (300, 20011, 64), (256, 40009, 32), (256, 70001, 20), (256, 140003, 128), (2100, 100, 7),
        (2100, 601, 64), (2100, 2003, 128), (2100, 7001, 20)]


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("rows,vocab,top", LONG)
def test_whole_rows(rows, vocab, top, dtype):
    """Rows enough that each has a workgroup (or a wave) of its own, at every length that a kernel is chosen by; a few
    of them, with special ones among these, against the definitions."""
    special = _special(vocab, dtype, 5)
    z = _logits(rows, vocab, dtype, 20)
    at = torch.linspace(0, rows - 1, len(special) + 4).long()
    z[at[:len(special)]] = special
    g = _gen(rows, vocab, 21)
    target = torch.randint(-1, vocab, (rows,), generator=g)
    ids, tz = _teacher(rows, vocab, top, dtype, 22)
    up = torch.randn(rows, generator=g)
    zd = _place(z, 1, 2)
    logp, ent, lse, tl, ti, stats = _score(zd, target, top, 1.3)
    sub = z[at]
    rl, rh, rs, el, eh, es = ref.logprobs(sub, target[at], 1.3)
    for got, want, bound in ((logp, rl, el), (ent, rh, eh), (lse, rs, es)):
        ref.near(got[at.to(DEV)], want, bound, torch.float32)
    assert torch.equal(ti.cpu()[at], ref.rank(sub)[:, :top])
    dz, ok = _guarded((rows, vocab), dtype)
    ql.qhead_logprobs_bwd(zd, target.to(DEV), stats, ent, up.to(DEV), None, dz, temperature=1.3)
    ref.near(dz[at.to(DEV)], *ref.logprobs_grad(sub, target[at], 1.3, up[at], None), dtype)
    assert ok()
    dev = lambda v: v.to(DEV)  # noqa: E731
    for t, alpha, label in ((2.0, 1.0, None), (2.0, 0.4, target), (1.0, 0.4, target)):
        want, grad, el, eg = ref.distill(sub, ids[at], tz[at], None if label is None else label[at], t, alpha, up[at])
        more = (dev(ids), dev(tz), None if label is None else dev(label))
        (loss, ok0), (dz, ok1) = _guarded((rows,), torch.float32), _guarded((rows, vocab), dtype)
        ql.qhead_distill_step(zd, *more, dev(up), loss, dz, temperature=t, alpha=alpha)
        ref.near(loss[at.to(DEV)], want, el, torch.float32)
        ref.near(dz[at.to(DEV)], grad, eg, dtype)
        assert ok0() and ok1()
        ql.qhead_distill_fwd(zd, *more, loss, temperature=t, alpha=alpha)
        ref.near(loss[at.to(DEV)], want, el, torch.float32)
        over = z.to(DEV)  # in place
        ql.qhead_distill_step(over, *more, dev(up), loss, over, temperature=t, alpha=alpha)
        assert torch.equal(over.nan_to_num(3.0), dz.nan_to_num(3.0))
