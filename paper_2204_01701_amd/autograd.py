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
"""
from __future__ import annotations

import torch

from . import (NEURON_TERMS, QL_BF16, QL_F32, QL_NEURON_QUADRA, QL_NEURON_T2, QL_NEURON_T24, conv_desc, epilogue,
               linear_desc, qlayer_conv2d_bwd_data, qlayer_conv2d_bwd_data_ex, qlayer_conv2d_bwd_relu,
               qlayer_conv2d_bwd_weight, qlayer_conv2d_fwd, qlayer_conv2d_fwd_ex,
               qlayer_linear_bwd, qlayer_linear_bwd_relu, qlayer_linear_fwd, qlayer_linear_fwd_ex,
               qhead_distill_bwd, qhead_distill_fwd, qhead_linear_bwd, qhead_linear_fwd, qhead_logprobs_bwd,
               qhead_logprobs_fwd)

__all__ = ["quad_conv2d", "quad_linear", "QuadConv2dFunction", "QuadLinearFunction", "linear_act", "token_logprobs",
           "distill_loss", "LinearActFunction", "TokenLogprobsFunction", "DistillLossFunction"]


def _qdtype(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return QL_BF16
    if t.dtype == torch.float32:
        return QL_F32
    raise TypeError(f"unsupported dtype {t.dtype}: use bfloat16 or float32")


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


def _terms(ws, nt):
    if any(w is None for w in ws[:nt]):
        raise ValueError(f"the neuron type has {nt} weighted terms")
    return list(ws[:nt]) + [None] * (3 - nt)


class QuadConv2dFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, wa, wb, wc, ba, bb, bc, stride, pad, recompute, neuron=QL_NEURON_QUADRA, relu=False,
                groups=1):
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
        ctx.save_for_backward(xn, *wn, *bl, ta, tb, y if relu else None)
        ctx.desc, ctx.recompute, ctx.has_bias, ctx.nt, ctx.neuron = d, recompute, b is not None, nt, neuron
        ctx.wdtype = wa.dtype
        return y.permute(0, 3, 1, 2)

    @staticmethod
    def backward(ctx, gy):
        d, nt = ctx.desc, ctx.nt
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
            return (dx, *dw, *db, None, None, None, None, None, None)
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
        return (dx, *dw, *db, None, None, None, None, None, None)


class QuadLinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, wa, wb, wc, ba, bb, bc, recompute, neuron=QL_NEURON_QUADRA, relu=False):
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
        ctx.save_for_backward(xc, *wl, *bl, ta, tb, y if relu else None)
        ctx.desc, ctx.recompute, ctx.has_bias, ctx.nt, ctx.neuron = d, recompute, b is not None, nt, neuron
        ctx.wdtype = wa.dtype
        return y

    @staticmethod
    def backward(ctx, gy):
        d, nt = ctx.desc, ctx.nt
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
            return (None,) * 10
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
        return (dx, *dw, *db, None, None, None)


def quad_conv2d(x, wa, wb=None, wc=None, ba=None, bb=None, bc=None, stride=1, pad=0, recompute=False,
                neuron=QL_NEURON_QUADRA, relu=False, groups=1):
    """Quadratic 2-D convolution layer (NCHW-shaped tensors, channels_last memory)."""
    return QuadConv2dFunction.apply(x, wa, wb, wc, ba, bb, bc, stride, pad, recompute, neuron, relu, groups)


def quad_linear(x, wa, wb=None, wc=None, ba=None, bb=None, bc=None, recompute=False, neuron=QL_NEURON_QUADRA,
                relu=False):
    """Quadratic fully-connected layer: x (B, I), weights (O, I)."""
    return QuadLinearFunction.apply(x, wa, wb, wc, ba, bb, bc, recompute, neuron, relu)


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
        raise RuntimeError("a gradient of linear_act, token_logprobs or distill_loss is differentiated: the library has no "
                           "kernels for these functions' second derivatives, they cannot be differentiated twice")


def _once(t, *of):
    """t, a gradient computed from `of`; where a graph is made of the backward (create_graph), tied to them in it: a
    tensor without a graph would pass for a constant there."""
    if t is None or not torch.is_grad_enabled() or not any(v is not None and v.requires_grad for v in of):
        return t
    return _Undifferentiable.apply(t, *of)


class LinearActFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, res, act, train=True):
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
            ctx.save_for_backward(xm, wm, z, x, w, b)  # (the last three for _once; no copies)
            ctx.act, ctx.xshape, ctx.wdtype = act, x.shape, w.dtype
            ctx.bdtype = b.dtype if b is not None else None
            ctx.rdtype = res.dtype if res is not None else None
        return y.view(shape)

    @staticmethod
    def backward(ctx, gy):
        x, w, z, *leaves = ctx.saved_tensors
        gx, gw, gb, gr = ctx.needs_input_grad[:4]
        dx = torch.empty(x.shape, device=x.device, dtype=x.dtype) if gx else None
        # (weights kept in float32 get the gradient as it was accumulated)
        dw = torch.empty(w.shape, device=x.device, dtype=x.dtype if ctx.wdtype is x.dtype else torch.float32) if gw else None
        db = torch.empty(w.shape[0], device=x.device) if gb else None
        if gx or gw or gb:
            qhead_linear_bwd(x, w, _matrix(gy), z, dx, dw, db, act=ctx.act)
        of = leaves if ctx.act != "none" else (None, None, None)  # through act'(z)
        return (_once(dx.view(ctx.xshape), gy, leaves[1], *of) if gx else None,
                _once(dw.to(ctx.wdtype), gy, leaves[0], *of) if gw else None,
                _once(db.to(ctx.bdtype), gy, *of) if gb else None, gy.to(ctx.rdtype) if gr else None, None, None)


def linear_act(x, weight, bias=None, residual=None, act="none"):
    """act(x weight^T + bias) + residual, with x (..., in), weight (out, in), bias (out), residual (..., out).

    act: "none", "relu", "gelu" (error function), "gelu_tanh" or "silu".  The product, the
    epilogue and the gradients run in the library's kernels in the dtype of x (the gradient of a
    float32 weight leaves them unrounded); the
    pre-activation is kept for the backward in that dtype where there is an activation and
    gradients are on (under no_grad and inference_mode it is not even written)."""
    # (inside an autograd function gradients are off, and its needs_input_grad does not know of no_grad)
    return LinearActFunction.apply(x, weight, bias, residual, act, torch.is_grad_enabled())


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
