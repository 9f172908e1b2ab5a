"""Linear layers in 8 bits for the weights that the optimizer owns.

The layers are compositions of the library's 8-bit operators (see `binding`: prm_rmsnorm_q8,
prm_quantize_q8, prm_matmul_q8 and the norm's gradient) as autograd functions.  Weights are stored
in x out, y = x @ W, as in the shape sets of `workloads`.

A step of training is

    y = norm_linear(x, residual, norm_weight, w8)     # or linear(x, w8)
    loss.backward()                                   # gradients in 8 bits, dW in the weight's type
    optimizer.step(...)                               # PeriodicRowwiseMuon on the weights
    w8.refresh()                                      # the weights' 8-bit codes again

What a layer keeps for its backward pass is one byte per element of its input.  Both products of the
backward pass run on 8-bit operands: the scales that run along a product's sum are folded into the
gradient before it is quantised, by row for dx = g W^T and by column for dW = x^T g.  The rounding to
8 bits is taken as the identity by the gradients (straight-through).  The gradients have no derivatives of
their own: a backward pass with create_graph=True is refused.
"""

from __future__ import annotations

import torch

from .binding import prm_matmul_q8, prm_quantize_q8, prm_rmsnorm_q8, prm_rmsnorm_q8_backward


class Weight8:
    """The 8-bit codes of a weight (in x out) with one scale for each output channel.  They are laid
    out once per change of the weight: call refresh() after each optimizer step."""

    def __init__(self, weight, format="int8"):
        self.weight = weight
        self.format = format
        self.refresh()

    def refresh(self):
        _, _, self.codes, self.scale = prm_quantize_q8(self.weight.detach(), by_rows=False, by_cols=True,
                                                       format=self.format)


def _refuse_second_derivative():
    # Gradient mode is on in a backward pass whose own graph is wanted.  A node that raises only when it is
    # differentiated would be passed by: the gradient's dependence on x and W runs through codes, not the graph.
    if torch.is_grad_enabled():
        raise RuntimeError("the 8-bit layers have no second derivatives: run backward without create_graph")


def _backward_products(grad_out, x8, sx, codes, scale, format, x_dtype, w_dtype, need_x, need_w):
    """(dx, dW) of y = (x8 * sx) @ (codes * scale), None for what is not needed."""
    gr, sr, gc, sc = prm_quantize_q8(grad_out, by_rows=need_x, by_cols=need_w, fold_rows=sx if need_w else None,
                                     fold_cols=scale if need_x else None, format=format)
    dx = prm_matmul_q8(gr, sr, codes.t(), None, out_dtype=x_dtype) if need_x else None
    dw = prm_matmul_q8(x8.t(), None, gc, sc, out_dtype=w_dtype) if need_w else None
    return dx, dw


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, w8):
        x8, sx, _, _ = prm_quantize_q8(x, format=w8.format)
        ctx.save_for_backward(x8, sx, w8.codes, w8.scale)
        ctx.format, ctx.types = w8.format, (x.dtype, weight.dtype)
        return prm_matmul_q8(x8, sx, w8.codes, w8.scale, out_dtype=x.dtype)

    @staticmethod
    def backward(ctx, grad_out):
        _refuse_second_derivative()
        x8, sx, codes, scale = ctx.saved_tensors
        need = ctx.needs_input_grad
        if not (need[0] or need[1]):
            return None, None, None
        dx, dw = _backward_products(grad_out, x8, sx, codes, scale, ctx.format, *ctx.types, need[0], need[1])
        return dx, dw, None


class _NormLinear(torch.autograd.Function):
    # x and residual come in the shape they were given: both get the same gradient, which autograd keeps apart
    # only where both get the same tensor, not two views of one.
    @staticmethod
    def forward(ctx, x, residual, norm_weight, weight, w8, eps):
        ctx.set_materialize_grads(False)
        ctx.shape = x.shape
        x = x.reshape(-1, x.shape[-1])
        if residual is not None:
            residual = residual.reshape(x.shape)
        x8, sx, h = prm_rmsnorm_q8(x, norm_weight, eps, residual=residual, format=w8.format)
        ctx.save_for_backward(x8, sx, w8.codes, w8.scale, x if h is None else h, norm_weight)
        ctx.format, ctx.eps, ctx.types = w8.format, eps, (x.dtype, weight.dtype)
        y = prm_matmul_q8(x8, sx, w8.codes, w8.scale, out_dtype=x.dtype)
        return y if h is None else (y, h)

    @staticmethod
    def backward(ctx, grad_out, grad_h=None):
        _refuse_second_derivative()
        x8, sx, codes, scale, h, norm_weight = ctx.saved_tensors
        need = ctx.needs_input_grad
        if grad_out is None:                # only the stream goes on; the caller may hold grad_h
            grad_h = grad_h.clone().reshape(ctx.shape)
            return (grad_h if need[0] else None, grad_h if need[1] else None, None, None, None, None)
        need_stream = need[0] or need[1] or need[2]
        if not (need_stream or need[3]):
            return (None,) * 6
        dy, dw = _backward_products(grad_out, x8, sx, codes, scale, ctx.format, *ctx.types, need_stream, need[3])
        dx = dn = None
        if need_stream:
            dx, dn = prm_rmsnorm_q8_backward(dy, h, norm_weight, ctx.eps, grad_h=grad_h)
            dx = dx.reshape(ctx.shape)
        return (dx if need[0] else None, dx if need[1] else None, dn if need[2] else None, dw, None, None)


def _as_given(y, x):
    return y.reshape(*x.shape[:-1], y.shape[-1])


def linear(x, w8):
    """x @ W in 8 bits: x (..., in), one vector too, bf16 or fp32, quantised by row; w8 a Weight8.  Returns (..., out) in
    x's type."""
    return _as_given(_Linear.apply(x.reshape(-1, x.shape[-1]), w8.weight, w8), x)


def norm_linear(x, residual, norm_weight, w8, eps=1e-6):
    """Root-mean-square norm of h = x + residual, then @ W, both in 8 bits: (y, h).  residual may be None
    (h = x); h carries the residual stream on."""
    if residual is None:
        return _as_given(_NormLinear.apply(x, None, norm_weight, w8.weight, w8, eps), x), x
    if residual.shape != x.shape:
        raise ValueError("x and residual must have the same shape")
    y, h = _NormLinear.apply(x, residual, norm_weight, w8.weight, w8, eps)
    return _as_given(y, x), _as_given(h, x)
