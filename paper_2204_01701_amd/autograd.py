"""Differentiable quadratic layers on top of the C ABI (arXiv 2204.01701).

``quad_conv2d`` and ``quad_linear`` are torch autograd functions whose
forward and backward run entirely in ``libqlayer.so``: the forward computes
Y = (W_a*X + b_a) o (W_b*X + b_b) + (W_c*X + b_c) (section 3.1,
eq:2ndneuron3), the backward the input, weight and bias gradients of
section 4.3 (eq:SD).  They offer the two memory modes of section 4.3:

* ``recompute=False`` (save): the forward keeps T_a = W_a*X + b_a and
  T_b = W_b*X + b_b for the backward;
* ``recompute=True`` (hybrid back-propagation): the forward keeps only X, and
  the backward regenerates T_a and T_b with the forward kernel (Y not
  written) before the gradient kernels.  The gradients are bitwise those of
  save mode, since the same kernel produces T_a and T_b in both.

``neuron`` selects the layer type (``QL_NEURON_*``): the proposed neuron or
one of the earlier designs of Table 1 (T4, T4 + identity, T3, T2, T2&4).  Weights
and biases of the terms a type lacks are passed as None.  T2 saves nothing
but X in either mode (its backward needs only X).

``relu=True`` applies the activation deeper networks put after each
quadratic layer (section 4.2, model construction) in the forward kernel's
epilogue; the backward is one library call that masks the incoming gradient
with y' > 0 and forms the layer's own gradients from it (no elementwise torch
operation).  ``groups`` (convolution): 1, or C for the
depth-wise setting (weights (C, 1, KH, KW)).

Layouts.  Convolution tensors are NCHW-shaped torch tensors; they are used in
channels_last memory format, whose memory is the library's NHWC (OHWI for
weights), so channels_last inputs are not copied and the outputs come back
channels_last.  X, the weights and Y share one dtype (bfloat16 or float32);
biases are float32 or None (all three or none).  Weight gradients are
returned in the weights' dtype, bias gradients in float32.

The end of a network: ``linear_act`` is a first-order fully-connected layer with bias,
activation and residual in one call, ``token_logprobs`` the log probabilities of
given tokens (class labels) with the entropy and the most likely alternatives,
``distill_loss`` the loss against a teacher's top logits, mixed with the label's
cross entropy.  They take leading dimensions of any kind.  Their gradients cannot be
differentiated again: under ``create_graph`` a second derivative through them raises.

A block trained with its activations in 8 bits: ``group_norm_act`` (group normalization
with an activation) and ``gated_linear`` (two projections, an activation, their product),
under the same terms.  They, ``linear_act`` and the quadratic layers take
``checkpoint="int8"``, the third memory mode beside saving and recomputing: what the backward
reads of the activations (X, T_a and T_b, pre-activations) is kept in 8 bits, blocks of 32
channels with a power of two each (include/qblock.h), and the gradients are formed from these
values.  A quadratic layer with relu=True keeps its output beside them, as it is, for the mask; where
that output is the next layer's X, the checkpoint of X comes on top of it.  The outputs are those without it, bit for bit (``gated_linear`` of up to 16 rows: but for a
rounding).  As nothing then ties the gradients to the
activations, a backward under ``create_graph`` raises.
"""
from __future__ import annotations

import math

import torch

from . import (NEURON_TERMS, QL_BF16, QL_F32, QL_NEURON_QUADRA, QL_NEURON_T2, QL_NEURON_T24, conv_desc, epilogue,
               linear_desc, qlayer_conv2d_bwd_data, qlayer_conv2d_bwd_data_ex, qlayer_conv2d_bwd_relu,
               qlayer_conv2d_bwd_weight, qlayer_conv2d_fwd, qlayer_conv2d_fwd_ex,
               qlayer_linear_bwd, qlayer_linear_bwd_relu, qlayer_linear_fwd, qlayer_linear_fwd_ex,
               qhead_distill_bwd, qhead_distill_fwd, qhead_linear_bwd, qhead_linear_fwd, qhead_logprobs_bwd,
               qhead_logprobs_fwd, BLOCK_KEEP, BlockGatedDesc, BlockKeepDesc, BlockNormDesc, HeadLinearDesc,
               _block_launch, _gated_fwd_query, _head_act, _int, _unaligned)

__all__ = ["quad_conv2d", "quad_linear", "QuadConv2dFunction", "QuadLinearFunction", "linear_act", "token_logprobs",
           "distill_loss", "LinearActFunction", "TokenLogprobsFunction", "DistillLossFunction", "group_norm_act",
           "gated_linear", "GroupNormActFunction", "GatedLinearFunction"]


def _qdtype(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return QL_BF16
    if t.dtype == torch.float32:
        return QL_F32
    raise TypeError(f"unsupported dtype {t.dtype}: use bfloat16 or float32")


def _tdtype(code: int) -> torch.dtype:
    return torch.bfloat16 if code == QL_BF16 else torch.float32


def _nhwc(t: torch.Tensor) -> torch.Tensor:
    """NCHW-shaped tensor -> contiguous NHWC view of its channels_last memory."""
    return t.contiguous(memory_format=torch.channels_last).permute(0, 2, 3, 1)


def _biases(ba, bb, bc, nt, O):
    bs = (ba, bb, bc)[:nt]
    if all(b is None for b in bs):
        return None
    if any(b is None for b in bs):
        raise ValueError("give the biases of every term of the neuron type or none")
    if any(b.numel() != O for b in bs):
        raise ValueError(f"each bias must have O = {O} elements")
    return [b.contiguous().float() for b in bs] + [None] * (3 - nt)


def _same_device(x, *others):
    """Every tensor on x's CUDA device (the kernels take raw device pointers)."""
    if x.device.type != "cuda":
        raise ValueError(f"the layer runs on a CUDA device; x is on {x.device}")
    for t in others:
        if t is not None and t.device != x.device:
            raise ValueError(f"every tensor must be on {x.device}; one is on {t.device}")


def _cast_grads(gs, dtype):
    """The float32 weight gradients (None: no such term) in the weights' dtype, in one launch."""
    if dtype == torch.float32:
        return gs
    src = [g for g in gs if g is not None]
    out = [torch.empty_like(g, dtype=dtype) for g in src]
    torch._foreach_copy_(out, src)
    return out + [None] * (len(gs) - len(out))


def _kept(checkpoint):
    """Whether activations are kept in 8 bits."""
    if checkpoint not in (None, "int8"):
        raise ValueError(f'checkpoint {checkpoint!r}: None or "int8" is required')
    return checkpoint is not None


def _no_graph():
    """Refuses create_graph where a checkpoint stands for an activation."""
    if torch.is_grad_enabled():
        raise RuntimeError('checkpoint="int8" keeps no activation that a gradient could be differentiated through: no backward '
                           "under create_graph, and none can be differentiated twice")


def _pack(t):
    """The 8-bit checkpoint (q, e) of a matrix or a dense tensor, in blocks of its last dimension (None: none)."""
    if t is None:
        return None, None
    cols = t.shape[-1]
    rows = t.numel() // cols
    q = torch.empty((rows, cols), device=t.device, dtype=torch.int8)
    e = torch.empty((rows, -(-cols // BLOCK_KEEP)), device=t.device, dtype=torch.uint8)
    ld = t.stride(0) if t.dim() == 2 and rows > 1 else cols
    _block_launch("qblock_pack8", BlockKeepDesc(rows, _int(cols), ld, _qdtype(t)), (t.data_ptr(), q.data_ptr(), e.data_ptr()), t.get_device())
    return q, e


# What a backward reads of its saved tensors it reads by their pointers.  A hook of the saved tensors may bring one back in
# another order of memory, or, by mistake, as something else than what was saved.

def _saved(t, what, dtype, shape, index):
    """A saved tensor whose dtype, shape and device are those that were saved."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        raise ValueError(f"the saved {what} came back as {t.dtype} {tuple(t.shape)} on {t.device}, {dtype} {tuple(shape)} on the "
                         "gradient's device was saved")
    return t


def _saved_dense(t, what, dtype, shape, index):
    """... and dense, row after row."""
    t = _saved(t, what, dtype, shape, index)
    return t if t.is_contiguous() else t.contiguous()


def _unpack(q, e, dtype, shape, index):
    """The values (`shape`, in blocks of its last dimension) of a saved checkpoint (None: none)."""
    if q is None:
        return None
    rows, cols = math.prod(shape[:-1]), shape[-1]
    q = _saved_dense(q, "checkpoint", torch.int8, (rows, cols), index)
    e = _saved_dense(e, "checkpoint's exponents", torch.uint8, (rows, -(-cols // BLOCK_KEEP)), index)
    t = torch.empty(shape, device=q.device, dtype=dtype)
    _block_launch("qblock_unpack8", BlockKeepDesc(rows, cols, cols, _qdtype(t)), (q.data_ptr(), e.data_ptr(), t.data_ptr()), index)
    return t


def _terms(ws, nt):
    if any(w is None for w in ws[:nt]):
        raise ValueError(f"the neuron type has {nt} weighted terms")
    return list(ws[:nt]) + [None] * (3 - nt)


class QuadConv2dFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, wa, wb, wc, ba, bb, bc, stride, pad, recompute, neuron=QL_NEURON_QUADRA, relu=False,
                groups=1, checkpoint=None):
        N, C, H, W = x.shape
        O, C2, KH, KW = wa.shape
        nt = NEURON_TERMS[neuron]
        ws = _terms((wa, wb, wc), nt)
        if C2 * groups != C or any(w.shape != wa.shape for w in ws[:nt]):
            raise ValueError("weight shapes must be (O, C / groups, KH, KW) for every term")
        _same_device(x, *ws, ba, bb, bc)
        d = conv_desc(N, C, H, W, O, KH, KW, stride, pad, _qdtype(x), neuron, groups=groups)
        xn = _nhwc(x)
        wn = [_nhwc(w.to(x.dtype)) if w is not None else None for w in ws]
        b = _biases(ba, bb, bc, nt, O)
        bl = b if b is not None else [None, None, None]
        y = torch.empty((N, d.ho, d.wo, O), device=x.device, dtype=x.dtype)
        recompute = recompute or neuron == QL_NEURON_T2  # (T2 saves nothing but X)
        ta = torch.empty_like(y) if not recompute else None
        tb = torch.empty_like(y) if not recompute and nt >= 2 else None
        if relu:
            qlayer_conv2d_fwd_ex(d, xn, *wn, *bl, y, ta, tb, epi=epilogue(relu=True))
        else:
            qlayer_conv2d_fwd(d, xn, *wn, *bl, y, ta, tb)
        # Everything the backward reads goes through save_for_backward, the
        # output y' (the ReLU mask) included: an in-place change of any of them
        # then fails the version check instead of silently changing the
        # gradients, and no reference cycle through ctx keeps them alive.
        ctx.kept = _kept(checkpoint) and any(ctx.needs_input_grad[:7])
        if ctx.kept:
            ctx.save_for_backward(*_pack(xn), *wn, *bl, *_pack(ta), *_pack(tb), y if relu else None)
        else:
            ctx.save_for_backward(xn, *wn, *bl, ta, tb, y if relu else None)
        ctx.desc, ctx.recompute, ctx.has_bias, ctx.nt, ctx.neuron = d, recompute, b is not None, nt, neuron
        ctx.wdtype = wa.dtype
        return y.permute(0, 3, 1, 2)

    @staticmethod
    def backward(ctx, gy):
        d, nt = ctx.desc, ctx.nt
        if ctx.kept:
            _no_graph()
            xq, xe, wa, wb, wc, ba, bb, bc, taq, tae, tbq, tbe, relu_y = ctx.saved_tensors
            y_shape = (d.n, d.ho, d.wo, d.o)
            index = gy.get_device()
            xn = _unpack(xq, xe, _tdtype(d.dtype), (d.n, d.h, d.w, d.c), index)
            ta, tb = (_unpack(q, e, xn.dtype, y_shape, index) for q, e in ((taq, tae), (tbq, tbe)))
        else:
            xn, wa, wb, wc, ba, bb, bc, ta, tb, relu_y = ctx.saved_tensors
        wn, bl = [wa, wb, wc], [ba, bb, bc]
        if ctx.neuron == QL_NEURON_T2:
            ta = xn  # its input gradient takes X in place of a saved map
        elif ctx.recompute:
            ta = torch.empty((d.n, d.ho, d.wo, d.o), device=xn.device, dtype=xn.dtype)
            tb = torch.empty_like(ta) if nt >= 2 else None
            qlayer_conv2d_fwd(d, xn, *wn, *bl, None, ta, tb)
        gyn = _nhwc(gy.to(xn.dtype))
        need_x, need_w = ctx.needs_input_grad[0], any(ctx.needs_input_grad[1:4])
        need_b = ctx.has_bias and any(ctx.needs_input_grad[4:7])
        dx = dw = db = None
        if relu_y is not None and (need_x or need_w or need_b):
            # the ReLU's mask and both gradients in one library call (G = gy o [y' > 0] formed once)
            dxn = torch.empty_like(xn) if need_x else None
            dwn = [torch.empty(wn[0].shape, device=xn.device, dtype=torch.float32) if i < nt else None
                   for i in range(3)] if (need_w or need_b) else [None, None, None]
            db = [torch.empty(d.o, device=xn.device, dtype=torch.float32) if i < nt else None
                  for i in range(3)] if need_b else None
            qlayer_conv2d_bwd_relu(d, xn, gyn, relu_y, None if ctx.neuron == QL_NEURON_T2 else ta, tb, *wn, dxn,
                                   *dwn, *(db or [None, None, None]))
            dx = dxn.permute(0, 3, 1, 2) if need_x else None
            dw = [g.permute(0, 3, 1, 2) if g is not None else None for g in _cast_grads(dwn, ctx.wdtype)]
            db = db or [None, None, None]
            return (dx, *dw, *db, *[None] * 7)
        if need_x:
            dxn = torch.empty_like(xn)
            if ctx.neuron == QL_NEURON_T24:  # (the chain rule through X o X needs X)
                qlayer_conv2d_bwd_data_ex(d, gyn, ta, tb, xn, *wn, dxn)
            else:
                qlayer_conv2d_bwd_data(d, gyn, ta, tb, *wn, dxn)
            dx = dxn.permute(0, 3, 1, 2)
        if need_w or need_b:
            dwn = [torch.empty(wn[0].shape, device=xn.device, dtype=torch.float32) if i < nt else None
                   for i in range(3)]
            db = [torch.empty(d.o, device=xn.device, dtype=torch.float32) if i < nt else None
                  for i in range(3)] if need_b else None
            qlayer_conv2d_bwd_weight(d, xn, gyn, None if ctx.neuron == QL_NEURON_T2 else ta, tb, *dwn,
                                     *(db or [None, None, None]))
            dw = [g.permute(0, 3, 1, 2) if g is not None else None for g in _cast_grads(dwn, ctx.wdtype)]
        dw = dw or [None, None, None]
        db = db or [None, None, None]
        return (dx, *dw, *db, *[None] * 7)


class QuadLinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, wa, wb, wc, ba, bb, bc, recompute, neuron=QL_NEURON_QUADRA, relu=False, checkpoint=None):
        if x.dim() != 2 or wa.dim() != 2:
            raise ValueError("x must be (B, I) and the weights (O, I)")
        B, I = x.shape
        O = wa.shape[0]
        nt = NEURON_TERMS[neuron]
        ws = _terms((wa, wb, wc), nt)
        if wa.shape[1] != I or any(w.shape != wa.shape for w in ws[:nt]):
            raise ValueError(f"weight shapes must be (O, {I}) for every term")
        _same_device(x, *ws, ba, bb, bc)
        d = linear_desc(B, I, O, _qdtype(x), neuron)
        xc = x.contiguous()
        wl = [w.to(x.dtype).contiguous() if w is not None else None for w in ws]
        b = _biases(ba, bb, bc, nt, O)
        bl = b if b is not None else [None, None, None]
        y = torch.empty((B, O), device=x.device, dtype=x.dtype)
        recompute = recompute or neuron == QL_NEURON_T2
        ta = torch.empty_like(y) if not recompute else None
        tb = torch.empty_like(y) if not recompute and nt >= 2 else None
        if relu:
            qlayer_linear_fwd_ex(d, xc, *wl, *bl, y, ta, tb, epi=epilogue(relu=True))
        else:
            qlayer_linear_fwd(d, xc, *wl, *bl, y, ta, tb)
        ctx.kept = _kept(checkpoint) and any(ctx.needs_input_grad[:7])
        if ctx.kept:
            ctx.save_for_backward(*_pack(xc), *wl, *bl, *_pack(ta), *_pack(tb), y if relu else None)
        else:
            ctx.save_for_backward(xc, *wl, *bl, ta, tb, y if relu else None)
        ctx.desc, ctx.recompute, ctx.has_bias, ctx.nt, ctx.neuron = d, recompute, b is not None, nt, neuron
        ctx.wdtype = wa.dtype
        return y

    @staticmethod
    def backward(ctx, gy):
        d, nt = ctx.desc, ctx.nt
        if ctx.kept:
            _no_graph()
            xq, xe, wa, wb, wc, ba, bb, bc, taq, tae, tbq, tbe, relu_y = ctx.saved_tensors
            index = gy.get_device()
            xc = _unpack(xq, xe, _tdtype(d.dtype), (d.batch, d.in_), index)
            ta, tb = (_unpack(q, e, xc.dtype, (d.batch, d.out), index) for q, e in ((taq, tae), (tbq, tbe)))
        else:
            xc, wa, wb, wc, ba, bb, bc, ta, tb, relu_y = ctx.saved_tensors
        wl, bl = [wa, wb, wc], [ba, bb, bc]
        if ctx.neuron == QL_NEURON_T2:
            pass  # the dense backward takes X itself
        elif ctx.recompute:
            ta = torch.empty((d.batch, d.out), device=xc.device, dtype=xc.dtype)
            tb = torch.empty_like(ta) if nt >= 2 else None
            qlayer_linear_fwd(d, xc, *wl, *bl, None, ta, tb)
        gyc = gy.to(xc.dtype).contiguous()
        need_x, need_w = ctx.needs_input_grad[0], any(ctx.needs_input_grad[1:4])
        need_b = ctx.has_bias and any(ctx.needs_input_grad[4:7])
        if not (need_x or need_w or need_b):
            return (None,) * 11
        dx = torch.empty_like(xc) if need_x else None
        dw = [torch.empty(wl[0].shape, device=xc.device, dtype=torch.float32) if i < nt else None
              for i in range(3)] if (need_w or need_b) else None
        db = [torch.empty(d.out, device=xc.device, dtype=torch.float32) if i < nt else None
              for i in range(3)] if need_b else None
        if relu_y is not None:  # the ReLU's mask and both gradients in one library call
            qlayer_linear_bwd_relu(d, xc, gyc, relu_y, ta, tb, *wl, dx, *(dw or [None] * 3), *(db or [None] * 3))
        else:
            qlayer_linear_bwd(d, xc, gyc, ta, tb, *wl, dx, *(dw or [None] * 3), *(db or [None] * 3))
        dw = _cast_grads(dw, ctx.wdtype) if dw is not None else [None, None, None]
        db = db or [None, None, None]
        return (dx, *dw, *db, *[None] * 4)


def quad_conv2d(x, wa, wb=None, wc=None, ba=None, bb=None, bc=None, stride=1, pad=0, recompute=False,
                neuron=QL_NEURON_QUADRA, relu=False, groups=1, checkpoint=None):
    """Quadratic 2-D convolution layer (NCHW-shaped tensors, channels_last memory).

    checkpoint="int8" keeps X and, unless recompute, T_a and T_b in 8 bits for the backward (with relu also the output, in full)."""
    _kept(checkpoint)
    return QuadConv2dFunction.apply(x, wa, wb, wc, ba, bb, bc, stride, pad, recompute, neuron, relu, groups,
                                    checkpoint if torch.is_grad_enabled() else None)


def quad_linear(x, wa, wb=None, wc=None, ba=None, bb=None, bc=None, recompute=False, neuron=QL_NEURON_QUADRA,
                relu=False, checkpoint=None):
    """Quadratic fully-connected layer: x (B, I), weights (O, I); checkpoint as in quad_conv2d."""
    _kept(checkpoint)
    return QuadLinearFunction.apply(x, wa, wb, wc, ba, bb, bc, recompute, neuron, relu,
                                    checkpoint if torch.is_grad_enabled() else None)


# --- the end of a network -----------------------------------------------------------

def _matrix(t):
    """(..., c) as a matrix whose rows are contiguous and do not overlap (a view where there is one)."""
    if t.dim() != 2:
        t = t.reshape(-1, t.shape[-1]) if t.numel() else t.new_empty((t.shape[:-1].numel(), t.shape[-1]))
    rows, cols = t.shape
    ld, step = t.stride()
    return t.contiguous() if (cols > 1 and step != 1) or (rows > 1 and ld < cols) else t


def _column(t, rows):
    """A gradient or target per row as a contiguous vector."""
    return (t if t.dim() == 1 else t.reshape(rows)).contiguous()


def _float_column(t, rows):
    t = _column(t, rows)
    return t if t.dtype is torch.float32 else t.float()


class _Undifferentiable(torch.autograd.Function):
    """A gradient as a function of what it was computed from, whose own derivative raises."""
    @staticmethod
    def forward(ctx, t, *of):
        return t.view_as(t)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("a gradient of linear_act, token_logprobs, distill_loss, group_norm_act or gated_linear is "
                           "differentiated: the library has no kernels for these functions' second derivatives, they cannot "
                           "be differentiated twice")


def _once(t, *of):
    """t, a gradient computed from `of`; where a graph is made of the backward (create_graph), tied to them in it: a
    tensor without a graph would pass for a constant there."""
    if t is None or not torch.is_grad_enabled() or not any(v is not None and v.requires_grad for v in of):
        return t
    return _Undifferentiable.apply(t, *of)


class LinearActFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, res, act, train=True, checkpoint=None):
        _same_device(x, w, b, res)
        if w.dim() != 2 or x.dim() < 1 or x.shape[-1] != w.shape[1]:
            raise ValueError(f"x (..., in) and w (out, in) are required, got {tuple(x.shape)} and {tuple(w.shape)}")
        if b is not None and b.shape != w.shape[:1]:
            raise ValueError(f"the bias must have {w.shape[0]} elements")
        shape = x.shape[:-1] + w.shape[:1]
        if res is not None and res.shape != shape:
            raise ValueError(f"the residual must have the output's shape {tuple(shape)}, got {tuple(res.shape)}")
        xm, wm = _matrix(x), _matrix(w.to(x.dtype))
        y = torch.empty((xm.shape[0], w.shape[0]), device=x.device, dtype=x.dtype)
        z = torch.empty_like(y) if train and act != "none" and any(ctx.needs_input_grad[:3]) else None
        qhead_linear_fwd(xm, wm, b.contiguous().float() if b is not None else None,
                         _matrix(res.to(x.dtype)) if res is not None else None, y, z, act=act)
        if train:
            ctx.kept = _kept(checkpoint)
            if ctx.kept:
                # (of x only what the weight's gradient reads)
                ctx.save_for_backward(*_pack(xm if ctx.needs_input_grad[1] else None), wm, *_pack(z))
            else:
                ctx.save_for_backward(xm, wm, z, x, w, b)  # (the last three for _once; no copies)
            ctx.act, ctx.xshape, ctx.wdtype = act, x.shape, w.dtype
            ctx.bdtype = b.dtype if b is not None else None
            ctx.rdtype = res.dtype if res is not None else None
        return y.view(shape)

    @staticmethod
    def backward(ctx, gy):
        gx, gw, gb, gr = ctx.needs_input_grad[:4]
        if ctx.kept:
            _no_graph()
            return LinearActFunction._kept_backward(ctx, gy)
        x, w, z, *leaves = ctx.saved_tensors
        dx = torch.empty(x.shape, device=x.device, dtype=x.dtype) if gx else None
        # (weights kept in float32 get the gradient as it was accumulated)
        dw = torch.empty(w.shape, device=x.device, dtype=x.dtype if ctx.wdtype is x.dtype else torch.float32) if gw else None
        db = torch.empty(w.shape[0], device=x.device) if gb else None
        if gx or gw or gb:
            qhead_linear_bwd(x, w, _matrix(gy), z, dx, dw, db, act=ctx.act)
        of = leaves if ctx.act != "none" else (None, None, None)  # through act'(z)
        return (_once(dx.view(ctx.xshape), gy, leaves[1], *of) if gx else None,
                _once(dw.to(ctx.wdtype), gy, leaves[0], *of) if gw else None,
                _once(db.to(ctx.bdtype), gy, *of) if gb else None, gy.to(ctx.rdtype) if gr else None, *[None] * 3)

    @staticmethod
    def _kept_backward(ctx, gy):
        xq, xe, w, zq, ze = ctx.saved_tensors
        gx, gw, gb, gr = ctx.needs_input_grad[:4]
        dtype, dev, index = gy.dtype, gy.device, gy.get_device()
        dx = dw = db = None
        if gx or gw or gb:
            dy = _matrix(gy)
            (m, n), k = dy.shape, ctx.xshape[-1]
            w = _matrix(_saved(w, "weight", dtype, (n, k), index))
            x, z = _unpack(xq, xe, dtype, (m, k), index) if gw else None, _unpack(zq, ze, dtype, (m, n), index)
            dx = torch.empty(ctx.xshape, device=dev, dtype=dtype) if gx else None
            dw = torch.empty((n, k), device=dev, dtype=dtype if ctx.wdtype is dtype else torch.float32) if gw else None
            db = torch.empty(n, device=dev) if gb else None
            px, pw, pdy = _ptr(x), w.data_ptr(), dy.data_ptr()
            desc = HeadLinearDesc(m, k, n, k, w.stride(0) if n > 1 else k, n, dy.stride(0) if m > 1 else n, _qdtype(w), _head_act(ctx.act),
                                  _unaligned(px, pw, pdy), gw and dw.dtype is not dtype)
            _block_launch("qhead_linear_bwd", desc, (px, pw, pdy, _ptr(z), _ptr(dx), _ptr(dw), _ptr(db)), index, "qhead_linear_bwd_workspace_size")
        return (dx, dw.to(ctx.wdtype) if gw else None, db.to(ctx.bdtype) if gb else None, gy.to(ctx.rdtype) if gr else None, *[None] * 3)


def linear_act(x, weight, bias=None, residual=None, act="none", checkpoint=None):
    """act(x weight^T + bias) + residual, with x (..., in), weight (out, in), bias (out), residual (..., out).

    act: "none", "relu", "gelu" (error function), "gelu_tanh" or "silu".  The product, the
    epilogue and the gradients run in the library's kernels in the dtype of x (the gradient of a
    float32 weight leaves them unrounded); the
    pre-activation is kept for the backward in that dtype where there is an activation and
    gradients are on (under no_grad and inference_mode it is not even written).  checkpoint="int8": x and the
    pre-activation are kept in 8 bits."""
    _kept(checkpoint)
    # (inside an autograd function gradients are off, and its needs_input_grad does not know of no_grad)
    return LinearActFunction.apply(x, weight, bias, residual, act, torch.is_grad_enabled(), checkpoint)


class TokenLogprobsFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, target, temperature, top, train=True):
        ctx.set_materialize_grads(False)
        lead = logits.shape[:-1]
        if target.shape != lead or target.dtype is not torch.int64:
            raise ValueError(f"target must be int64 of shape {tuple(lead)}, got {target.dtype} {tuple(target.shape)}")
        z = _matrix(logits)
        rows, dev = z.shape[0], z.device
        t = _column(target, rows)
        logp, entropy = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
        stats = torch.empty((rows, 2), device=dev) if train and ctx.needs_input_grad[0] else None
        top_logp = torch.empty((rows, top), device=dev) if top else None
        top_ids = torch.empty((rows, top), device=dev, dtype=torch.int64) if top else None
        qhead_logprobs_fwd(z, t, logp, entropy, None, top_logp, top_ids, stats, temperature)
        if stats is not None:
            ctx.temperature, ctx.shape = temperature, logits.shape
            ctx.save_for_backward(z, t, stats, entropy, logits)
        out = (logp, entropy) if len(lead) == 1 else (logp.view(lead), entropy.view(lead))
        if not top:
            return out
        more = top_logp.view(lead + (top,)), top_ids.view(lead + (top,))
        ctx.mark_non_differentiable(*more)
        return out + more

    @staticmethod
    def backward(ctx, g, h, *_):
        if g is None and h is None:
            return None, None, None, None, None
        z, t, stats, entropy, logits = ctx.saved_tensors
        rows, of = z.shape[0], (g, h, logits)
        g = _float_column(g, rows) if g is not None else torch.zeros(rows, device=z.device)
        h = _float_column(h, rows) if h is not None else None
        dz = torch.empty(z.shape, device=z.device, dtype=z.dtype)
        qhead_logprobs_bwd(z, t, stats, entropy.view(rows), g, h, dz, ctx.temperature)
        return _once(dz if dz.shape == ctx.shape else dz.view(ctx.shape), *of), None, None, None, None


def token_logprobs(logits, target, temperature=1.0, top=0):
    """(log probability of `target`, entropy) under softmax(logits / temperature), float32.

    logits (..., vocab); target (...) int64, negative where there is none (log probability 0, no
    gradient from it).  top > 0 adds (top_logp, top_ids) of shape (..., top): the most likely
    tokens, equal logits by rising id (no gradient passes through them)."""
    return TokenLogprobsFunction.apply(logits, target, temperature, top, torch.is_grad_enabled())


class DistillLossFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, t_ids, t_logits, labels, temperature, alpha, train=True):
        lead = logits.shape[:-1]
        if (t_ids is not None and t_ids.shape[:-1] != lead) or (t_logits is not None and t_logits.shape[:-1] != lead):
            raise ValueError(f"the teacher's places do not fit logits of shape {tuple(logits.shape)}")
        if labels is not None and labels.shape != lead:
            raise ValueError(f"labels: shape {tuple(labels.shape)}, expected {tuple(lead)}")
        z = _matrix(logits)
        rows, dev = z.shape[0], z.device
        if t_ids is not None and t_logits is not None:
            if t_ids.dim() != 2:
                t_ids, t_logits = (v.reshape(rows, v.shape[-1]) for v in (t_ids, t_logits))
            if t_logits.dtype is not z.dtype:
                t_logits = t_logits.float()  # (float32 as it is: only what the caller rounded is rounded)
            t_ids, t_logits = t_ids.contiguous(), t_logits.contiguous()
        if labels is not None:
            labels = _column(labels, rows)
        loss = torch.empty(rows, device=dev)
        stats = torch.empty((rows, 4), device=dev) if train and ctx.needs_input_grad[0] else None
        qhead_distill_fwd(z, t_ids, t_logits, labels, loss, stats, temperature, alpha)
        if stats is not None:
            ctx.save_for_backward(z, t_ids, t_logits, labels, stats, logits)
            ctx.how, ctx.shape = (temperature, alpha), logits.shape
        return loss if len(lead) == 1 else loss.view(lead)

    @staticmethod
    def backward(ctx, g):
        z, ids, tz, labels, stats, logits = ctx.saved_tensors
        dz = torch.empty(z.shape, device=z.device, dtype=z.dtype)
        qhead_distill_bwd(z, ids, tz, labels, stats, _float_column(g, z.shape[0]), dz, *ctx.how)
        return _once(dz if dz.shape == ctx.shape else dz.view(ctx.shape), g, logits), None, None, None, None, None, None


def distill_loss(logits, teacher_ids, teacher_logits, labels=None, temperature=1.0, alpha=1.0):
    """Per-row loss of a student against a teacher's top logits, float32:

        alpha T^2 KL(q || softmax(logits / T)) + (1 - alpha) cross_entropy(logits, label),

    q the softmax of teacher_logits / T over the row's places.  logits (..., vocab); teacher_ids int64
    (negative: an empty place) and teacher_logits (..., K), or both None: float32 ones, as token_logprobs gives
    them, are taken in float32 whatever the dtype of the logits; labels (...) int64, negative
    where a row has none, or None.  The gradient goes to the logits."""
    return DistillLossFunction.apply(logits, teacher_ids, teacher_logits, labels, temperature, alpha, torch.is_grad_enabled())


# --- blocks trained with activations in 8 bits ----------------------------------------

def _dense_image(t):
    """t with its values in channels-last order, dense (4 dimensions), or row after row (2)."""
    return t.contiguous(memory_format=torch.channels_last) if t.dim() == 4 else t.contiguous()


def _f32(t):
    return t if t is None or (t.dtype is torch.float32 and t.is_contiguous()) else t.contiguous().float()


def _ptr(t):
    return None if t is None else t.data_ptr()


class GroupNormActFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, act, train=True, checkpoint=None):
        _same_device(x, weight, bias)
        if x.dim() not in (2, 4):
            raise ValueError(f"x (N, C, H, W) or (N, C) is required, got {tuple(x.shape)}")
        n, c = x.shape[:2]
        hw = 1 if x.dim() == 2 else x.shape[2] * x.shape[3]
        if not isinstance(groups, int) or groups < 1 or c < 1 or c % groups or hw < 1:
            raise ValueError(f"{groups!r} groups of {c} channels and {hw} pixels: a whole number that divides the channels is required")
        if (weight is not None and weight.shape != (c,)) or (bias is not None and bias.shape != (c,)):
            raise ValueError(f"weight and bias must have {c} elements")
        xn = _dense_image(x)
        gamma, beta = _f32(weight), _f32(bias)
        y = torch.empty_like(xn)
        desc = BlockNormDesc(_int(n), _int(hw), _int(c), groups, _qdtype(x), _head_act(act), eps)
        stats = q = e = mean = rstd = None
        train = train and any(ctx.needs_input_grad[:3])
        kept = train and _kept(checkpoint)
        if train:
            stats = torch.empty((2, n, groups), device=x.device)
            mean = stats.data_ptr()
            rstd = mean + 4 * n * groups
        if kept:
            q = torch.empty((n * hw, c), device=x.device, dtype=torch.int8)
            e = torch.empty((n * hw, -(-c // BLOCK_KEEP)), device=x.device, dtype=torch.uint8)
        _block_launch("qblock_norm_fwd", desc, (xn.data_ptr(), _ptr(gamma), _ptr(beta), y.data_ptr(), mean, rstd, _ptr(q), _ptr(e)),
                      x.get_device(), "qblock_norm_fwd_workspace_size")
        if train:
            if kept:
                ctx.save_for_backward(q, e, gamma, beta, stats)
            else:
                ctx.save_for_backward(xn, gamma, beta, stats, x, weight, bias)  # (the last three for _once; no copies)
            ctx.desc, ctx.kept = desc, kept
            ctx.dtypes = None if weight is None else weight.dtype, None if bias is None else bias.dtype
        return y

    @staticmethod
    def backward(ctx, gy):
        x = q = e = None
        of = ()
        gx, gw, gb = ctx.needs_input_grad[:3]
        desc = ctx.desc
        n, c, index = desc.n, desc.c, gy.get_device()
        if ctx.kept:
            _no_graph()
            q, e, gamma, beta, stats = ctx.saved_tensors
            q = _saved_dense(q, "checkpoint", torch.int8, (n * desc.hw, c), index)
            e = _saved_dense(e, "checkpoint's exponents", torch.uint8, (n * desc.hw, -(-c // BLOCK_KEEP)), index)
        else:
            x, gamma, beta, stats, *of = ctx.saved_tensors
            x = _dense_image(_saved(x, "input", gy.dtype, gy.shape, index))
        gamma, beta = (None if t is None else _saved_dense(t, "weight or bias", torch.float32, (c,), index) for t in (gamma, beta))
        stats = _saved_dense(stats, "statistics", torch.float32, (2, n, desc.groups), index)
        dy = _dense_image(gy)
        dx = torch.empty_like(dy) if gx else None
        dgamma = torch.empty(c, device=dy.device) if gw else None
        dbeta = torch.empty(c, device=dy.device) if gb else None
        mean = stats.data_ptr()
        _block_launch("qblock_norm_bwd", desc, (dy.data_ptr(), _ptr(x), _ptr(q), _ptr(e), _ptr(gamma), _ptr(beta), mean,
                                                mean + 4 * n * desc.groups, _ptr(dx), _ptr(dgamma), _ptr(dbeta)),
                      index, "qblock_norm_bwd_workspace_size")
        if gw and ctx.dtypes[0] is not torch.float32:
            dgamma = dgamma.to(ctx.dtypes[0])
        if gb and ctx.dtypes[1] is not torch.float32:
            dbeta = dbeta.to(ctx.dtypes[1])
        if torch.is_grad_enabled():
            dx, dgamma, dbeta = (_once(t, gy, *of) for t in (dx, dgamma, dbeta))
        return dx, dgamma, dbeta, None, None, None, None, None


def group_norm_act(x, groups, weight=None, bias=None, eps=1e-5, act="none", checkpoint=None):
    """act(weight (x - mean) / sqrt(var + eps) + bias), mean and variance over the pixels and channels of each group.

    x (N, C, H, W), used in channels_last memory, or (N, C); weight and bias (C) or None; act as in linear_act.
    The backward reads x, or with checkpoint="int8" what 8 bits of it say."""
    _kept(checkpoint)
    # (laid out here, where the copy has a graph of its own: inside, the backward would keep the copy, and x for _once)
    return GroupNormActFunction.apply(_dense_image(x), weight, bias, groups, eps, act, torch.is_grad_enabled(), checkpoint)


class GatedLinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, wg, wu, bg, bu, act, train=True, checkpoint=None):
        _same_device(x, wg, wu, bg, bu)
        if wg.dim() != 2 or x.dim() < 1 or x.shape[-1] != wg.shape[1] or wu.shape != wg.shape:
            raise ValueError(f"x (..., in) and two weights (out, in) are required, got {tuple(x.shape)}, {tuple(wg.shape)} and "
                             f"{tuple(wu.shape)}")
        if (bg is not None and bg.shape != wg.shape[:1]) or (bu is not None and bu.shape != wg.shape[:1]):
            raise ValueError(f"each bias must have {wg.shape[0]} elements")
        dtype, dev = x.dtype, x.device
        xm, wgm, wum = _matrix(x), _matrix(wg.to(dtype)), _matrix(wu.to(dtype))
        if wgm.stride() != wum.stride():
            wgm, wum = wgm.contiguous(), wum.contiguous()
        (m, k), n = xm.shape, wg.shape[0]
        h = torch.empty((m, n), device=dev, dtype=dtype)
        train = train and any(ctx.needs_input_grad[:5])
        kept = train and _kept(checkpoint)
        z = torch.empty((2, m, n), device=dev, dtype=dtype) if train and not kept else None
        q = e = None
        if kept:
            q = torch.empty((2, m, n), device=dev, dtype=torch.int8)
            e = torch.empty((2, m, -(-n // BLOCK_KEEP)), device=dev, dtype=torch.uint8)
        bgf, buf = _f32(bg), _f32(bu)
        ldx, ldw = (xm.stride(0) if m > 1 else k), (wgm.stride(0) if n > 1 else k)
        px, pg, pu = xm.data_ptr(), wgm.data_ptr(), wum.data_ptr()
        desc = BlockGatedDesc(_int(m), _int(k), _int(n), ldx, ldw, n, _qdtype(x), _head_act(act), _unaligned(px, pg, pu), 0)
        _block_launch("qblock_gated_fwd", desc, (px, pg, pu, _ptr(bgf), _ptr(buf), h.data_ptr(), _ptr(z), _ptr(q), _ptr(e)), x.get_device(),
                      _gated_fwd_query(m, q))
        if train:
            # (of x only what the weights' gradients read)
            xs = xm if any(ctx.needs_input_grad[1:3]) else None
            if kept:
                ctx.save_for_backward(*_pack(xs), wgm, wum, q, e)
            else:
                ctx.save_for_backward(xs, wgm, wum, z, x, wg, wu, bg, bu)  # (the last five for _once; no copies)
            ctx.kept, ctx.act, ctx.xshape, ctx.dtypes = kept, act, x.shape, [None if t is None else t.dtype for t in (wg, wu, bg, bu)]
        return h if x.dim() == 2 else h.view(x.shape[:-1] + (n,))

    @staticmethod
    def backward(ctx, gh):
        x = z = q = e = None
        of = ()
        gx, gwg, gwu, gbg, gbu = ctx.needs_input_grad[:5]
        gw = gwg or gwu
        dtype, dev, index = gh.dtype, gh.device, gh.get_device()
        dh = _matrix(gh)
        (m, n), k = dh.shape, ctx.xshape[-1]
        if ctx.kept:
            _no_graph()
            xq, xe, wg, wu, q, e = ctx.saved_tensors
            q = _saved_dense(q, "checkpoint", torch.int8, (2, m, n), index)
            e = _saved_dense(e, "checkpoint's exponents", torch.uint8, (2, m, -(-n // BLOCK_KEEP)), index)
            if gw:
                x = _unpack(xq, xe, dtype, (m, k), index)
        else:
            x, wg, wu, z, *of = ctx.saved_tensors
            z = _saved_dense(z, "projections", dtype, (2, m, n), index)
            x = _matrix(_saved(x, "input", dtype, (m, k), index)) if gw else None
        wg, wu = (_matrix(_saved(w, "weight", dtype, (n, k), index)) for w in (wg, wu))
        if wg.stride() != wu.stride():
            wg, wu = wg.contiguous(), wu.contiguous()
        # (weights kept in float32 get the gradient as it was accumulated)
        wdtype = dtype if ctx.dtypes[0] is dtype and ctx.dtypes[1] is dtype else torch.float32
        dx = torch.empty(ctx.xshape, device=dev, dtype=dtype) if gx else None
        dwg = torch.empty((n, k), device=dev, dtype=wdtype) if gw else None
        dwu = torch.empty((n, k), device=dev, dtype=wdtype) if gw else None
        dbg = torch.empty(n, device=dev) if gbg else None
        dbu = torch.empty(n, device=dev) if gbu else None
        px, pg, pu = _ptr(x), wg.data_ptr(), wu.data_ptr()
        desc = BlockGatedDesc(m, k, n, x.stride(0) if x is not None and m > 1 else k, wg.stride(0) if n > 1 else k,
                              dh.stride(0) if m > 1 else n, _qdtype(wg), _head_act(ctx.act), _unaligned(px, pg, pu), wdtype is not dtype)
        _block_launch("qblock_gated_bwd", desc, (px, pg, pu, dh.data_ptr(), _ptr(z), _ptr(q), _ptr(e), _ptr(dx), _ptr(dwg), _ptr(dwu),
                                                 _ptr(dbg), _ptr(dbu)), index, "qblock_gated_bwd_workspace_size")
        out = [dx, dwg if gwg else None, dwu if gwu else None, dbg, dbu]
        for i, d in enumerate(ctx.dtypes, 1):
            if out[i] is not None and out[i].dtype is not d:
                out[i] = out[i].to(d)
        if torch.is_grad_enabled():
            out = [_once(t, gh, *of) for t in out]
        return (*out, None, None, None)


def gated_linear(x, w_gate, w_up, b_gate=None, b_up=None, act="silu", checkpoint=None):
    """act(x w_gate^T + b_gate) * (x w_up^T + b_up), with x (..., in), weights (out, in), biases (out).

    Both projections, the activation (as in linear_act) and the product run in one kernel in the dtype of x.  The projections
    are kept for the backward in that dtype, or, and x with them, in 8 bits under checkpoint="int8"."""
    _kept(checkpoint)
    return GatedLinearFunction.apply(x, w_gate, w_up, b_gate, b_up, act, torch.is_grad_enabled(), checkpoint)
