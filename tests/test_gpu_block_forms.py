"""Group norm in every form that its plan may choose, by sizes and by the plan's overrides, against the definitions: registers of
2, 8 and 16 pixels a thread, chunks of one pass and of several, groups in parts, channels taken by 1, 2, 4 and 8, workgroups that
take several batches of samples."""
import pytest
import torch

import block_ref as ref
import paper_2204_01701_amd as ql
from test_gpu_block_keep import DEV, TYPES, type_ids
from test_gpu_block_norm import backward, forward, inputs

pytestmark = pytest.mark.gpu
types = pytest.mark.parametrize("dtype", TYPES, ids=type_ids)


@pytest.fixture
def plan(monkeypatch):
    def force(**how):
        for name, value in how.items():
            monkeypatch.setenv("QBLOCK_NORM_" + name, str(value))
    return force


def few_blocks(n, p, c):
    """Whether the checkpoint's definition, a loop over its blocks, is quick."""
    return n * p * -(-c // 32) < 4000


def both(n, p, c, groups, dtype):
    keep = few_blocks(n, p, c)
    forward(n, p, c, groups, dtype, "silu", keep=keep)
    backward(n, p, c, groups, dtype, "gelu")
    backward(n, p, c, groups, dtype, "silu", keep=keep, affine=False, offset=1)


@types
@pytest.mark.parametrize("fused", [0, 1], ids=["chunks", "registers"])
@pytest.mark.parametrize("p", [40, 300, 1500])
@pytest.mark.parametrize("cpg", [1, 2, 3, 4, 6, 8, 24])
def test_channels_of_a_group(cpg, p, fused, dtype, plan):
    plan(FUSED=fused)
    both(3, p, 9 * cpg, 9, dtype)


@types
@pytest.mark.parametrize("line", [32, 64, 128])
@pytest.mark.parametrize("p", [20, 70, 500])
@pytest.mark.parametrize("cpg", [1, 2, 4, 8])
def test_segments(cpg, p, line, dtype, plan):
    plan(FUSED=1, LINE=line)
    both(2, p, 20 * cpg, 20, dtype)


@pytest.mark.parametrize("cpg", [3, 6, 4, 8])
def test_sixteen_pixels_a_thread(cpg, plan):
    plan(FUSED=1, LINE=128)  # (segments of 32 channels in float32: 128 pixels at once, 12 of them a thread)
    forward(2, 1500, 9 * cpg, 9, torch.float32, "gelu")
    forward(2, 1500, 9 * cpg, 9, torch.float32, "none", affine=False, offset=1)


@types
@pytest.mark.parametrize("cpg", [1, 2, 4, 8])
def test_long_chunks(cpg, dtype, plan):
    plan(FUSED=0, WGS=2)  # (chunks of many passes: a mean of the first pixels, then differences to it)
    both(2, 3001, 7 * cpg, 7, dtype)
    forward(1, 9000, 64 * cpg, 64, dtype, "gelu")


@types
@pytest.mark.parametrize("cpg", [4101, 4102, 4100, 4104, 2049])
@pytest.mark.parametrize("n,p", [(2, 3), (1, 150)])
def test_groups_in_parts(n, p, cpg, dtype, plan):
    plan(FUSED=0)
    both(n, p, 2 * cpg, 2, dtype)


@types
@pytest.mark.parametrize("kept", [False, True], ids=["x", "int8"])
@pytest.mark.parametrize("how,n,p,c,groups", [
    # (two to five batches a workgroup)
    (dict(FUSED=0), 10000, 1, 3, 3), (dict(FUSED=0), 10000, 1, 2, 1), (dict(FUSED=0), 10000, 1, 4, 1), (dict(FUSED=0), 10000, 1, 8, 1),
    (dict(FUSED=1), 3000, 300, 1, 1), (dict(FUSED=1), 3000, 300, 2, 1), (dict(FUSED=1), 3000, 300, 4, 1), (dict(FUSED=1), 10000, 17, 24, 3),
    (dict(FUSED=1, LINE=32), 18, 300, 2048, 2048), (dict(FUSED=1, LINE=32), 18, 300, 2048, 256), (dict(FUSED=0), 5, 1, 255 * 4101, 255)])
def test_many_batches(how, n, p, c, groups, kept, dtype, plan):
    """Sums over batches: a dy whose mean is not 0, so that a lost or doubled batch shows in dgamma and dbeta."""
    plan(**how)
    x, gamma, beta, dy = inputs(n, p, c, dtype)
    dy = (dy.float() + 0.5).to(dtype)
    stats = ref.norm(x, groups, gamma, beta, 1e-5, "none")
    mean, rstd = (stats[k][0].float() for k in ("mean", "rstd"))
    given, dev = {}, [t.to(DEV) for t in (gamma, beta, mean, rstd)]
    xd = x.to(DEV)
    if kept:
        q, e = torch.empty(n * p, c, device=DEV, dtype=torch.int8), torch.empty(n * p, -(-c // 32), device=DEV, dtype=torch.uint8)
        ql.qblock_pack8(xd.view(n * p, c), q, e)
        x = ref.unpack(q.cpu(), e.cpu()).view(n, p, c)
        given, xd = dict(q=q, e=e), None
    dx, dg, db = torch.empty(n, p, c, device=DEV, dtype=dtype), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    ql.qblock_norm_bwd(dy.to(DEV), xd, groups, *dev, dx, dg, db, act="silu", **given)
    want = ref.norm_grads(dy, x, groups, gamma, beta, mean, rstd, "silu")
    for name, t in (("dx", dx), ("dgamma", dg), ("dbeta", db)):
        ref.near(t, *want[name], t.dtype)
