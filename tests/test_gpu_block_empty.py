"""Batches of no rows where only some gradients are wanted."""
import pytest
import torch

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
