"""Batches of no rows where only some gradients are wanted."""
import ctypes

import pytest
import torch

import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import gated_linear, group_norm_act, linear_act
from test_gpu_block_keep import DEV, TYPES, type_ids

pytestmark = pytest.mark.gpu
checkpoints = pytest.mark.parametrize("checkpoint", [None, "int8"])
types = pytest.mark.parametrize("dtype", TYPES, ids=type_ids)


@types
@checkpoints
@pytest.mark.parametrize("shape", [(0, 16, 3, 3), (0, 16)])
def test_group_norm_without_parameters(shape, checkpoint, dtype):
    x = torch.empty(shape, device=DEV, dtype=dtype, requires_grad=True)
    y = group_norm_act(x, 4, act="gelu", checkpoint=checkpoint)
    dx, = torch.autograd.grad(y, x, torch.empty_like(y))
    assert y.shape == dx.shape == x.shape


@types
@checkpoints
@pytest.mark.parametrize("shape", [(0, 40), (2, 0, 40)])
def test_gated_layer_with_frozen_weights(shape, checkpoint, dtype):
    x = torch.empty(shape, device=DEV, dtype=dtype, requires_grad=True)
    w, u = (torch.randn(33, 40, device=DEV, dtype=dtype) for _ in range(2))
    h = gated_linear(x, w, u, checkpoint=checkpoint)
    dx, = torch.autograd.grad(h, x, torch.empty_like(h))
    assert h.shape == shape[:-1] + (33,) and dx.shape == x.shape


@types
@checkpoints
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("shape", [(0, 40), (2, 0, 40)])
def test_first_order_layer_with_a_frozen_weight(shape, act, checkpoint, dtype):
    x = torch.empty(shape, device=DEV, dtype=dtype, requires_grad=True)
    w = torch.randn(33, 40, device=DEV, dtype=dtype)
    y = linear_act(x, w, act=act, checkpoint=checkpoint)
    dx, = torch.autograd.grad(y, x, torch.empty_like(y))
    assert y.shape == shape[:-1] + (33,) and dx.shape == x.shape


@types
def test_gated_weight_gradients_beside_a_buffer_for_the_inputs(dtype):
    """A caller of the C ABI whose dx is a buffer for larger batches: nothing is written there, the rest are zeros."""
    k, n = 24, 40
    dx, dwg, dwu = (torch.full((n, k), 77.0, device=DEV, dtype=dtype) for _ in range(3))
    dbg, dbu = (torch.full((n,), 77.0, device=DEV) for _ in range(2))
    d = ctypes.byref(ql.BlockGatedDesc(0, k, n, k, k, n, ql.QL_BF16 if dtype == torch.bfloat16 else ql.QL_F32, 4, 0, 0))
    need = ql.lib().qblock_gated_bwd_workspace_size(d)
    ws = torch.empty(max(need, 16), device=DEV, dtype=torch.uint8)
    status = ql.lib().qblock_gated_bwd(d, None, dwg.data_ptr(), dwu.data_ptr(), None, None, None, None,
                                       *(t.data_ptr() for t in (dx, dwg, dwu, dbg, dbu)), ws.data_ptr(), need,
                                       torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == 0 and bool((dx == 77).all())
    for t in (dwg, dwu, dbg, dbu):
        assert not t.any()
