"""What stands around a layer's products in training, as autograd functions: dropout, layer norm, the loss of a
linear head (see `binding`: prm_dropout, prm_layernorm, prm_head_loss and their gradients).

    draws = Draws(seed)
    y, h = layer_norm(x, weight, bias, residual=h, p=0.1, draws=draws)    # h = dropout(x) + h, y its norm
    u = linear(y, w8)                                                     # q8, or any product
    loss = head_loss(y, head, labels).sum() / count                      # softmax cross entropy, logits not kept
    loss.backward()
    optimizer.step(...)
    draws.advance()                                                       # other masks in the next step

No mask and no logits are kept: a mask is drawn again by the backward pass, the logits are computed again.  A step may be
captured into a graph, advance() with it; each replay then draws anew.  (As with any function of torch: no eager graph of
the same leaves may be alive while a backward pass is captured.)  The gradients have no derivatives of their own: a
backward pass with create_graph=True is refused.

The head's products wait for copies with a limit.  A wait that has run out is not seen by the call: binding.prm_q8_status(), which
waits for the device, says so; ask it now and then, at the latest before weights are written out.
"""

from __future__ import annotations

import torch

from .binding import (prm_dropout, prm_head_loss, prm_head_loss_backward, prm_layernorm, prm_layernorm_backward)


class Draws:
    """Where dropout takes its numbers from: a seed, and a counter on the device.  Every call of a step takes the next
    number; advance() ends the step, after its backward pass (which reads the counter again, and refuses to run if it has been
    advanced since).  Ranks that are to draw masks of their own need seeds of their own.

    A part of the forward pass that is run again in the backward pass has to take the numbers that it took at first:

        y = torch.utils.checkpoint.checkpoint(block, x, use_reentrant=False, context_fn=draws.checkpoint)

    Without that a call inside a backward pass is refused: it would draw a mask that the loss has not seen."""

    def __init__(self, seed, device="cuda"):
        self.seed = int(seed)
        self.counter = torch.zeros(1, dtype=torch.int64, device=device)
        self.calls = 0
        self._again = 0

    def take(self):
        if not self._again and torch._C._current_graph_task_id() >= 0:
            raise RuntimeError("a forward pass that is run again in a backward pass would draw other masks: "
                               "give the checkpoint use_reentrant=False and context_fn=draws.checkpoint")
        self.calls += 1
        return self.calls - 1

    def advance(self):
        self.counter.add_(self.calls)
        self.calls = 0

    def checkpoint(self):
        """The two contexts of torch.utils.checkpoint's context_fn: the second one's calls take the first one's numbers."""
        first = _First(self)
        return first, _Again(first)


class _First:
    def __init__(self, draws):
        self.draws = draws

    def __enter__(self):
        self.calls, self.version = self.draws.calls, self.draws.counter._version

    def __exit__(self, *_):
        return None


class _Again:
    def __init__(self, first):
        self.first = first
        self.kept = []

    def __enter__(self):
        draws = self.first.draws
        if draws.counter._version != self.first.version:
            raise RuntimeError("the counter has been advanced since the forward pass that is run again")
        self.kept.append(draws.calls)
        draws.calls = self.first.calls
        draws._again += 1

    def __exit__(self, *_):
        draws = self.first.draws
        draws.calls = self.kept.pop()
        draws._again -= 1


def _refuse_second_derivative():
    if torch.is_grad_enabled():
        raise RuntimeError("these layers have no second derivatives: run backward without create_graph")


def _rows(t, cols):
    return None if t is None else t.reshape(t.shape[:-1].numel(), cols)        # cols may be 0


def _result(t, shape):
    """An operator's rows in the shape of what went in.  Not as a view: autograd forbids writing to a view that a function
    of its own returns (a caller's relu_, say), and follows what is written to this."""
    return t.reshape(shape).detach()


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, offset, counter):
        ctx.save_for_backward(counter)
        ctx.draw = p, seed, offset
        cols = x.shape[-1]
        return _result(prm_dropout(_rows(x, cols), p, seed, offset, counter, _rows(residual, cols)), x.shape)

    @staticmethod
    def backward(ctx, grad):
        _refuse_second_derivative()
        counter, = ctx.saved_tensors
        grad_x = None
        if ctx.needs_input_grad[0]:
            grad_x = prm_dropout(_rows(grad, grad.shape[-1]), *ctx.draw, counter).reshape(grad.shape)
        return grad_x, grad if ctx.needs_input_grad[1] else None, None, None, None, None


class _LayerNorm(torch.autograd.Function):
    # Gradients of x and residual that are the same come as the same tensor: two views of one autograd would add up in place.
    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps, add_one, p, seed, offset, counter):
        ctx.set_materialize_grads(False)
        cols = x.shape[-1]
        x2 = _rows(x, cols)
        y, h, mean, rstd = prm_layernorm(x2, weight, bias, eps, residual=_rows(residual, cols), add_one=add_one, p=p, seed=seed,
                                         offset=offset, counter=counter)
        ctx.save_for_backward(x2 if h is None else h, mean, rstd, weight, counter)
        ctx.how = add_one, p, seed, offset
        ctx.shape = x.shape
        y = _result(y, x.shape)
        return y if h is None else (y, _result(h, x.shape))

    @staticmethod
    def backward(ctx, grad_y, grad_h=None):
        _refuse_second_derivative()
        h, mean, rstd, weight, counter = ctx.saved_tensors
        add_one, p, seed, offset = ctx.how
        need = ctx.needs_input_grad
        cols = h.shape[1]
        if grad_y is None:
            if grad_h is None:
                return (None,) * 10
            grad_r = grad_h.clone()             # the caller may hold grad_h
            grad_x = grad_r
            if p > 0 and need[0]:
                grad_x = prm_dropout(_rows(grad_h, cols), p, seed, offset, counter).reshape(ctx.shape)
            grad_w = grad_b = None
        else:
            grad_x, grad_r, grad_w, grad_b = prm_layernorm_backward(
                _rows(grad_y, cols), h, mean, rstd, weight, grad_h=_rows(grad_h, cols), add_one=add_one, p=p, seed=seed,
                offset=offset, counter=counter, need_weight=need[2], need_bias=need[3])
            grad_x = grad_x.reshape(ctx.shape)
            grad_r = grad_x if grad_r is None else grad_r.reshape(ctx.shape)
        return (grad_x if need[0] else None, grad_r if need[1] else None, grad_w, grad_b) + (None,) * 6


class _HeadLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, labels):
        loss, lse = prm_head_loss(x, weight, labels)
        ctx.save_for_backward(x, weight, labels, lse)
        return loss

    @staticmethod
    def backward(ctx, grad_loss):
        _refuse_second_derivative()
        x, weight, labels, lse = ctx.saved_tensors
        grad_x, grad_w = prm_head_loss_backward(grad_loss, x, weight, labels, lse, need_x=ctx.needs_input_grad[0],
                                                need_weight=ctx.needs_input_grad[1])
        return grad_x, grad_w, None


def _number(p, draws):
    """(seed, offset, counter) of one call."""
    if p == 0:
        return 0, 0, None
    if draws is None:
        raise ValueError("dropout needs draws")
    return draws.seed, draws.take(), draws.counter


def dropout(x, p, draws, residual=None):
    """x (..., cols), bf16 or fp32, with its elements dropped with probability p and the others divided by 1 - p, plus residual."""
    if residual is not None and residual.shape != x.shape:
        raise ValueError("x and residual must have the same shape")
    if p == 0:
        return x if residual is None else x + residual
    return _Dropout.apply(x, residual, p, *_number(p, draws))


def layer_norm(x, weight=None, bias=None, eps=1e-6, residual=None, p=0.0, draws=None, add_one=False):
    """Layer norm over the last dimension of h = dropout(x, p) + residual: (y, h).  h is x itself without either.

    weight and bias: cols, or groups x cols, a row for each part of the rows of x (..., cols) cut into `groups` equal ones
    (scale and shift of each sample of a batch); both in one shape and type, a bias without a weight: cols.  add_one takes 1 + weight."""
    if residual is not None and residual.shape != x.shape:
        raise ValueError("x and residual must have the same shape")
    out = _LayerNorm.apply(x, residual, weight, bias, eps, add_one, p, *_number(p, draws))
    return out if isinstance(out, tuple) else (out, x)


def head_loss(x, weight, labels):
    """Softmax cross entropy of the logits x @ weight for labels (...): fp32 losses of labels' shape, 0 where a label is not in
    0..vocab-1 (such a row has no part in the gradients, whatever it holds).  x (..., d), weight d x vocab,
    or the transposed view of an embedding, both bf16."""
    if labels.shape != x.shape[:-1]:
        raise ValueError("labels must have x's shape without its last dimension")
    return _HeadLoss.apply(x.reshape(-1, x.shape[-1]), weight, labels.reshape(-1)).reshape(labels.shape)
