"""The first-order layer with pointers off the 16-byte vector and the workspace of a caller that did not announce
them: the C entry points alone, since the binding announces by itself; against float64."""
import ctypes

import pytest
import torch

import head_ref as ref
import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("m,k,n", [(1, 64, 40), (130, 256, 264), (600, 1024, 768)])
def test_misaligned_pointers_that_are_not_announced(m, k, n, dtype):
    """`unaligned` 0 and a workspace for that: no copies, the same accuracy."""
    g = torch.Generator().manual_seed(75)
    x, w, dy, z = (torch.randn(s, generator=g).to(dtype) for s in ((m, k), (n, k), (m, n), (m, n)))

    def off(t):
        wide = torch.full((t.numel() + 1,), float("nan"), dtype=dtype)
        wide[1:] = t.flatten()
        return wide.to(DEV)[1:].view(t.shape)

    xd, wd, dyd, zd = (off(t) for t in (x, w, dy, z))
    code = ql.QL_BF16 if dtype == BF else ql.QL_F32
    d = ctypes.byref(ql.HeadLinearDesc(m, k, n, k, k, n, n, code, ql.HEAD_ACTS["silu"], 0, 0))
    y, dx, dw, db = (torch.empty(s, device=DEV, dtype=t) for s, t in (((m, n), dtype), ((m, k), dtype), ((n, k), dtype), ((n,), torch.float32)))
    L, st = ql.lib(), torch.cuda.current_stream().cuda_stream
    for query, call, ptrs in ((L.qhead_linear_fwd_workspace_size, L.qhead_linear_fwd, (xd, wd, None, None, y, None)),
                              (L.qhead_linear_bwd_workspace_size, L.qhead_linear_bwd, (xd, wd, dyd, zd, dx, dw, db))):
        need = query(d)
        ws = torch.empty(need + 16, dtype=torch.uint8, device=DEV)
        ws[need:] = 77
        assert call(d, *(None if t is None else t.data_ptr() for t in ptrs), ws.data_ptr(), need, st) == 0
        assert bool((ws[need:] == 77).all())
    ry, _, ey, _ = ref.linear(x, w, None, None, "silu")
    ref.near(y, ry, ey, dtype)
    want = ref.linear_grads(x, w, dy, z, "silu")
    for name, got in (("dx", dx), ("dw", dw), ("db", db)):
        ref.near(got, *want[name], got.dtype)
