"""Checkpoints in 8 bits against their definition, bit for bit: both types, odd rows, strides and alignments, zeros, the ends of
the range, NaN and infinities; guards around the outputs."""
import math

import pytest
import torch

import block_ref as ref
import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float32]
type_ids = ["bf16", "fp32"]


def rows_of(t, offset, pad, foreign=math.nan):
    """t on the GPU as rows of a wider tensor, `offset` elements from its start."""
    wide = torch.full((t.shape[0], offset + t.shape[1] + pad), foreign, dtype=t.dtype)
    wide[:, offset:offset + t.shape[1]] = t
    return wide.to(DEV)[:, offset:offset + t.shape[1]]


def guarded(shape, dtype, fill=77):
    n = math.prod(shape)
    raw = torch.full((n + 131,), fill, dtype=dtype, device=DEV)
    return raw[67:67 + n].view(shape), lambda: bool((raw[:67] == fill).all() and (raw[67 + n:] == fill).all())


def _check(x, offset=0, pad=0):
    rows, cols = x.shape
    q, okq = guarded((rows, cols), torch.int8)
    e, oke = guarded((rows, -(-cols // 32)), torch.uint8)
    ql.qblock_pack8(rows_of(x, offset, pad), q, e)
    rq, re, x8 = ref.pack(x)
    assert torch.equal(e.cpu(), re) and torch.equal(q.cpu(), rq)
    for dtype in TYPES:
        back, ok = guarded((rows, cols), dtype)
        ql.qblock_unpack8(q, e, back)
        got = back.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(x8)) and torch.equal(got.nan_to_num(3.0), x8.nan_to_num(3.0))
        wide = rows_of(torch.zeros(rows, cols, dtype=dtype), offset, pad, 5.0)
        ql.qblock_unpack8(q, e, wide)
        assert torch.equal(wide.double().cpu().nan_to_num(3.0), x8.nan_to_num(3.0))
        base = wide._base if wide._base is not None else wide
        assert bool((base[:, :offset] == 5).all() and (base[:, offset + cols:] == 5).all())
        assert ok()
    assert okq() and oke()


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (1, 8), (5, 31), (4, 32), (4, 33), (2, 64), (7, 100), (70, 65), (9, 1000), (300, 3)])
def test_against_the_definition(rows, cols, dtype):
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp(2 * torch.randn(rows, cols, generator=g))
    x[torch.rand(rows, generator=g) < 0.2] = 0
    x = x.to(dtype)
    _check(x)
    _check(x, 1, 2)
    _check(x, 8, 8)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
def test_ends_of_the_range(dtype):
    f = torch.finfo(dtype)
    x = torch.zeros(16, 40, dtype=torch.float64)
    x[0, 0], x[1, 3], x[2, :] = f.max, -f.max, f.max
    x[3, 5], x[4, 39], x[5, 1] = math.inf, math.nan, -math.inf
    x[6, :], x[7, 2], x[8, 1] = f.tiny, f.tiny * 127, f.tiny * f.eps  # (the last is subnormal)
    x[9, :] = torch.arange(40) - 20.5  # halves at a step of 1
    x[9, 31] = 127
    x[10, :], x[11, :] = -0.0, 1e-30
    x[12, :] = torch.exp2(torch.arange(40).double() - 20)
    x[13, :2] = torch.tensor([f.max, f.max / 128])
    x[14, 0], x[15, 0] = 127 * 2.0**20, 127.5 * 2.0**20
    _check(x.to(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
def test_no_rows_and_many(dtype):
    ql.qblock_pack8(torch.empty(0, 5, device=DEV, dtype=dtype), torch.empty(0, 5, device=DEV, dtype=torch.int8),
                    torch.empty(0, 1, device=DEV, dtype=torch.uint8))
    # more blocks than a launch's threads take at once: the whole against the packed rows by themselves
    x = torch.randn(2**20 + 3, 96, device=DEV).to(dtype)[:, :65]
    q, e = torch.empty(x.shape, device=DEV, dtype=torch.int8), torch.empty(x.shape[0], 3, device=DEV, dtype=torch.uint8)
    ql.qblock_pack8(x, q, e)
    for rows in (slice(0, 5), slice(2**20 - 2, 2**20 + 3)):
        rq, re, _ = ref.pack(x[rows].cpu())
        assert torch.equal(q[rows].cpu(), rq) and torch.equal(e[rows].cpu(), re)
    back = torch.empty(x.shape, device=DEV, dtype=dtype)
    ql.qblock_unpack8(q, e, back)
    blocks = torch.nn.functional.pad(x.float(), (0, 31)).view(-1, 3, 32).abs().amax(2)
    step = torch.exp2(e.float() - 127)
    # the least exponent: half the step would not do.  A block of zeros alone has the least of all, -126, whatever half of it
    # would do; a block of one value, as the rows' last are here, is a zero now and then
    assert bool((step * 127 >= blocks).all() and ((step * 63.5 < blocks) | (blocks == 0)).all())
    assert bool((e[blocks == 0] == 1).all())
    assert bool(((back.float() - x.float()).abs() <= step.repeat_interleave(32, 1)[:, :65] / 2).all())


WRONG = [lambda t, i, u: ql.qblock_pack8(t(4, 40), i(4, 41), u(4, 2)), lambda t, i, u: ql.qblock_pack8(t(4, 40), i(4, 40), u(4, 1)),
         lambda t, i, u: ql.qblock_pack8(t(4, 40), u(4, 40), u(4, 2)), lambda t, i, u: ql.qblock_pack8(t(4, 40), i(4, 80)[:, :40], u(4, 2)),
         lambda t, i, u: ql.qblock_pack8(t(40, 4).t(), i(4, 40), u(4, 2)), lambda t, i, u: ql.qblock_unpack8(i(4, 40), u(5, 2), t(4, 40)),
         lambda t, i, u: ql.qblock_unpack8(i(4, 40), u(4, 2), t(1, 40).expand(4, 40)), lambda t, i, u: ql.qblock_pack8(t(4, 40), None, u(4, 2)),
         lambda t, i, u: ql.qblock_pack8(t(4, 40).half(), i(4, 40), u(4, 2)), lambda t, i, u: ql.qblock_pack8(t(4, 40), i(4, 40).cpu(), u(4, 2))]


@pytest.mark.parametrize("k", range(len(WRONG)))
def test_wrong_tensors(k):
    def t(*s):
        return torch.zeros(*s, device=DEV)

    def i(*s):
        return torch.zeros(*s, device=DEV, dtype=torch.int8)

    def u(*s):
        return torch.zeros(*s, device=DEV, dtype=torch.uint8)

    with pytest.raises(ValueError):
        WRONG[k](t, i, u)


def test_on_another_stream():
    st, x = torch.cuda.Stream(), torch.randn(1000, 96, device=DEV)
    q, e = torch.empty(x.shape, device=DEV, dtype=torch.int8), torch.empty(1000, 3, device=DEV, dtype=torch.uint8)
    torch.cuda.synchronize()
    ql.qblock_pack8(x, q, e, stream=st)
    st.synchronize()
    rq, re, _ = ref.pack(x[:20].cpu())
    assert torch.equal(q[:20].cpu(), rq) and torch.equal(e[:20].cpu(), re)
