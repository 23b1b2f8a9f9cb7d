"""Device memory that the gated layer takes beside its tensors while it serves a few rows."""
import pytest
import torch

import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import gated_linear
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
