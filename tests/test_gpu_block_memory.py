"""Device memory: what the gated layer takes beside its tensors while it serves a few rows, what group norm keeps for its backward."""
import pytest
import torch

import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import gated_linear, group_norm_act
from test_gpu_block_keep import DEV

pytestmark = pytest.mark.gpu


def taken(f):
    """Bytes that a call holds at its highest beyond what it returns."""
    f()
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out = f()
    peak = torch.cuda.max_memory_allocated() - before
    return peak - (torch.cuda.memory_allocated() - before), out


@pytest.mark.parametrize("m", [1, 16])
@pytest.mark.parametrize("k,offset", [(1025, 0), (1024, 1)], ids=["odd rows", "misaligned"])
def test_a_few_rows_take_no_workspace(m, k, offset):
    """Weights that a product of many rows would copy: read in place."""
    n, rows = 2048, torch.randn(16, k, device=DEV, dtype=torch.bfloat16)
    wg, wu = (torch.randn(n * k + offset, device=DEV, dtype=torch.bfloat16)[offset:].view(n, k) for _ in range(2))
    x, h = rows[:m], torch.empty(m, n, device=DEV, dtype=torch.bfloat16)
    with torch.no_grad():
        extra, got = taken(lambda: gated_linear(x, wg, wu))
    assert extra == 0
    for stream in (None, torch.cuda.current_stream()):
        extra, _ = taken(lambda: ql.qblock_gated_fwd(x, wg, wu, None, None, h, stream=stream))
        assert extra == 0 and torch.equal(h, got)


@pytest.mark.parametrize("checkpoint,maps", [(None, 1), ("int8", 0.6)])
@pytest.mark.parametrize("layout", [torch.contiguous_format, torch.channels_last], ids=["NCHW", "NHWC"])
def test_group_norm_keeps_its_input_once(layout, checkpoint, maps):
    """Between forward and backward: one map (33/64 of one in 8 bits), whatever the order in which it came."""
    x = torch.randn(16, 64, 64, 64, device=DEV, dtype=torch.bfloat16).contiguous(memory_format=layout).requires_grad_(True)
    g, b = (torch.randn(64, device=DEV, requires_grad=True) for _ in range(2))
    size = x.numel() * 2
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    h = x * 1  # (an activation that only the layer holds)
    y = group_norm_act(h, 8, g, b, act="silu", checkpoint=checkpoint)
    del h
    assert torch.cuda.memory_allocated() - before <= (1 + maps) * size + (1 << 20)
    dx, _, _ = torch.autograd.grad(y, (x, g, b), torch.ones_like(y))
    assert dx.shape == x.shape
