"""More than 2^31 values, more rows than a launch's threads take: what lies behind the ends of 32-bit counters."""
import pytest
import torch

import block_ref as ref
import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_checkpoint_of_long_rows():
    """Three rows of 2^30 + 40 values: the end of the last one."""
    rows, cols = 3, 2**30 + 40
    x = torch.zeros(rows, cols, device=DEV, dtype=torch.bfloat16)
    end = torch.randn(rows, 72).bfloat16()
    x[:, -72:] = end.to(DEV)
    q = torch.empty(rows, cols, device=DEV, dtype=torch.int8)
    e = torch.empty(rows, -(-cols // 32), device=DEV, dtype=torch.uint8)
    ql.qblock_pack8(x, q, e)
    rq, re, x8 = ref.pack(end)  # (2^30 + 40 - 72 is a multiple of 32: the blocks are the same)
    assert torch.equal(q[:, -72:].cpu(), rq) and torch.equal(e[:, -3:].cpu(), re)
    assert int(q[:, :-72].count_nonzero()) == 0 and bool((e[:, :-3] == 1).all())
    x.fill_(7)
    ql.qblock_unpack8(q, e, x)
    assert torch.equal(x[:, -72:].double().cpu(), x8) and int(x[:, :-72].count_nonzero()) == 0


@pytest.mark.parametrize("n,hw,c,groups", [(2, 1200000, 1024, 4), (5000000, 7, 64, 8), (70000000, 1, 32, 4)])
def test_group_norm(n, hw, c, groups):
    """A sample at the end, against the same sample by itself in float64."""
    x = torch.randn(n, hw, c, device=DEV, dtype=torch.bfloat16)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, groups, device=DEV), torch.empty(n, groups, device=DEV)
    ql.qblock_norm_fwd(x, groups, None, None, y, mean, rstd, act="silu")
    last = x[-1].view(hw, groups, c // groups).double()
    m = last.mean(dim=(0, 2))
    d = last - m[:, None]
    r = torch.rsqrt((d * d).mean(dim=(0, 2)) + 1e-5)
    # (sums in partial sums of up to 320 roundings, of values up to 6 around 0)
    assert (mean[-1].double() - m).abs().max() <= 320 * 2.0**-24
    assert ((rstd[-1].double() - r) / r).abs().max() <= 320 * 2.0**-24
    want = torch.nn.functional.silu(d * r[:, None]).view(hw, c)
    got = y[-1].double()
    assert ((got - want).abs() <= 2.0**-8 * want.abs() + 1e-4).all()
    del want, got, d
    # the backward over the same map: dx of the last sample, and the parameters' gradients of a dy of one
    y.fill_(0)
    y[-1] = 1
    dx, dg, db = torch.empty_like(x), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    ql.qblock_norm_bwd(y, x, groups, None, None, mean, rstd, dx, dg, db)
    assert int(dx[0].count_nonzero()) == 0
    xh = ((last - mean[-1].double()[:, None]) * rstd[-1].double()[:, None])
    assert torch.equal(db, torch.full_like(db, hw)) or (db - hw).abs().max() <= 320 * 2.0**-24 * hw
    assert (dg.double() - xh.sum(0).view(c)).abs().max() <= 320 * 2.0**-24 * xh.abs().sum(0).max()
    # t is 1 throughout: dx = -rstd xh avg(xh), and avg(t) - 1 = 0, each to its roundings
    assert dx[-1].abs().max() <= 320 * 2.0**-24 * float(r.max()) * (1 + float(xh.abs().max()) ** 2)


def test_gated_layer():
    """2^24 + 9 rows onto 160: more than 2^31 values in h and its halves; the last rows, and the gradients of the weights."""
    m, k, n = 2**24 + 9, 24, 160
    x = torch.randn(m, k, device=DEV, dtype=torch.bfloat16)
    wg, wu = (torch.randn(n, k, device=DEV).div(5).bfloat16() for _ in range(2))
    h, z = torch.empty(m, n, device=DEV, dtype=torch.bfloat16), torch.empty(2, m, n, device=DEV, dtype=torch.bfloat16)
    ql.qblock_gated_fwd(x, wg, wu, None, None, h, z)
    want = ref.gated(x[-300:].cpu(), wg.cpu(), wu.cpu(), None, None, "silu")
    ref.near(h[-300:], *want["h"], torch.bfloat16)
    for i, name in enumerate("gu"):
        ref.near(z[i, -300:], *want[name], torch.bfloat16)
    h.fill_(0)
    dh = torch.randn(300, n).bfloat16()
    h[-300:] = dh.to(DEV)
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    dbg, dbu = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ql.qblock_gated_bwd(x, wg, wu, h, z, dx, dwg, dwu, dbg, dbu)
    want = ref.gated_grads(x[-300:].cpu(), wg.cpu(), wu.cpu(), dh, *z[:, -300:].cpu(), "silu", torch.bfloat16)
    for name, t in (("dx", dx[-300:]), ("dwg", dwg), ("dwu", dwu), ("dbg", dbg), ("dbu", dbu)):
        ref.near(t, *want[name], t.dtype)
    assert int(dx[:-300].count_nonzero()) == 0
