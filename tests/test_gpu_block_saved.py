"""Hooks of the saved tensors that bring them back in another order of memory: the gradients are those without the hook, bit for
bit; tensors that come back on another device or of another dtype are refused before a kernel reads them."""
import pytest
import torch

from paper_2204_01701_amd.autograd import gated_linear, group_norm_act, linear_act, quad_conv2d, quad_linear
from test_block_saved_cpu import ORDERS
from test_gpu_block_keep import DEV, TYPES, type_ids

pytestmark = pytest.mark.gpu


def check(leaves, f, order):
    """Gradients of f(*leaves) with every saved tensor brought back as `order` leaves it, against those without."""
    y = f(*leaves)
    dy = torch.randn_like(y)
    want = torch.autograd.grad(y, leaves, dy)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, order):
        y = f(*leaves)
    for got, w in zip(torch.autograd.grad(y, leaves, dy), want):
        assert torch.equal(got, w)


def refused(leaves, f):
    for wrong in (lambda t: t.cpu(), lambda t: t.half()):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, wrong):
            y = f(*leaves)
        with pytest.raises(ValueError):
            torch.autograd.grad(y, leaves, torch.randn_like(y))


def leaf(*shape, dtype):
    return torch.randn(*shape, device=DEV).to(dtype).requires_grad_(True)


def _gpu_order(order):
    """The orders of the CPU's tests on tensors of this device."""
    if order.__name__ == "spread":
        def spread(t):
            wide = torch.zeros(*t.shape, 2, dtype=t.dtype, device=t.device)
            wide[..., 0] = t
            return wide[..., 0]
        return spread
    return order


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("checkpoint", [None, "int8"])
@pytest.mark.parametrize("m,k,n", [(33, 40, 72), (9, 17, 5)])
def test_gated_layer(m, k, n, checkpoint, order, dtype):
    leaves = [leaf(m, k, dtype=dtype), leaf(n, k, dtype=dtype), leaf(n, k, dtype=dtype)]

    def f(*leaves):
        return gated_linear(*leaves, checkpoint=checkpoint)
    if checkpoint is None:
        check(leaves, f, _gpu_order(order))
    else:  # (the weights and the projections' checkpoint; x's own is read by unpack8, the input's gradient alone does not need it)
        x, wg, wu = leaves
        check([x], lambda x: gated_linear(x, wg.detach(), wu.detach(), checkpoint=checkpoint), _gpu_order(order))
    refused(leaves, f)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("checkpoint", [None, "int8"])
@pytest.mark.parametrize("shape", [(3, 36, 5, 7), (9, 36)])
def test_group_norm(shape, checkpoint, order, dtype):
    leaves = [leaf(*shape, dtype=dtype), leaf(36, dtype=torch.float32), leaf(36, dtype=dtype)]

    def f(x, g, b):
        return group_norm_act(x, 4, g, b, act="silu", checkpoint=checkpoint)
    check(leaves, f, _gpu_order(order))
    refused(leaves, f)


def of_checkpoints(order):
    """The hook for the checkpoints' tensors alone."""
    return lambda t: order(t) if t.dtype in (torch.int8, torch.uint8) else t


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layer", ["linear", "gated", "quadratic", "convolution"])
def test_checkpoints(layer, order, dtype):
    def leaves(*shapes):
        return [leaf(*s, dtype=dtype) for s in shapes]
    if layer == "convolution":
        of, f = leaves((2, 40, 5, 6), *[(36, 40, 3, 3)] * 3), lambda *a: quad_conv2d(*a, pad=1, checkpoint="int8")
    elif layer == "quadratic":
        of, f = leaves((20, 40), *[(36, 40)] * 3), lambda *a: quad_linear(*a, checkpoint="int8")
    elif layer == "gated":
        of, f = leaves((20, 40), (36, 40), (36, 40)), lambda *a: gated_linear(*a, checkpoint="int8")
    else:
        of, f = leaves((20, 40), (36, 40)), lambda *a: linear_act(*a, act="gelu", checkpoint="int8")
    check(of, f, of_checkpoints(_gpu_order(order)))
    for wrong in (lambda t: t.cpu(), lambda t: t.short()):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, of_checkpoints(wrong)):
            y = f(*of)
        with pytest.raises(ValueError):
            torch.autograd.grad(y, of, torch.randn_like(y))


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("m,k,n", [(33, 40, 72), (9, 17, 5)])
def test_first_order_layer(m, k, n, order, dtype):
    leaves = [leaf(m, k, dtype=dtype), leaf(n, k, dtype=dtype)]

    def f(*leaves):
        return linear_act(*leaves, act="silu", checkpoint="int8")
    check(leaves, f, _gpu_order(order))
    refused(leaves, f)
    x, w = leaves  # (the weight alone: the input's gradient without an activation reads nothing else)
    check([x], lambda x: linear_act(x, w.detach(), checkpoint="int8"), _gpu_order(order))
    refused([x], lambda x: linear_act(x, w.detach(), checkpoint="int8"))


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("checkpoint", [None, "int8"])
@pytest.mark.parametrize("pinned", [False, True])
def test_kept_in_host_memory(pinned, checkpoint, dtype):
    """torch's own hook, whose pinned copies are dense whatever was saved."""
    def of(*shapes):
        return [leaf(*s, dtype=dtype) for s in shapes]
    wide = torch.randn(36, 96, device=DEV).to(dtype)
    halves = [wide[:, i:i + 40].requires_grad_(True) for i in (0, 48)]  # (one row stride, other than their length)
    image = torch.randn(2, 40, 5, 6, device=DEV).to(dtype).contiguous(memory_format=torch.channels_last).requires_grad_(True)
    for leaves, f in ((of((20, 40)) + halves, lambda *a: gated_linear(*a, checkpoint=checkpoint)),
                      (of((20, 40)) + halves[:1], lambda *a: linear_act(*a, act="gelu", checkpoint=checkpoint)),
                      ([image, *of((40,), (40,))], lambda x, g, b: group_norm_act(x, 4, g, b, act="silu", checkpoint=checkpoint)),
                      (of((20, 40), *[(36, 40)] * 3), lambda *a: quad_linear(*a, relu=True, checkpoint=checkpoint)),
                      ([image, *of(*[(36, 40, 3, 3)] * 3)], lambda *a: quad_conv2d(*a, pad=1, relu=True, checkpoint=checkpoint))):
        y = f(*leaves)
        dy = torch.randn_like(y)
        want = torch.autograd.grad(y, leaves, dy)
        with torch.autograd.graph.save_on_cpu(pin_memory=pinned):
            y = f(*leaves)
        for got, w in zip(torch.autograd.grad(y, leaves, dy), want):
            assert torch.equal(got, w)
