"""Dropout in a forward pass that is run again in the backward pass: the same numbers, or a refusal.  On the CPU the draws are taken by
the tests' own form of dropout."""

import pytest
import torch
from torch.utils.checkpoint import checkpoint

import train_reference as R
from paper_2608_20818_b200 import layers as L


def host_dropout(x, p, seed, offset=0, counter=None, residual=None, stream=None):
    out = R.dropped(x.float(), p, seed, offset + int(counter))
    return (out if residual is None else out + residual.float()).to(x.dtype)


@pytest.fixture(params=["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cpu":
        monkeypatch.setattr(L, "prm_dropout", host_dropout)
    return request.param


def model(x, draws, block):
    """Calls before, inside (twice) and behind what is run again."""
    h = L.dropout(x, 0.5, draws)
    for _ in range(2):
        h = block(lambda t: L.dropout(torch.sin(L.dropout(torch.tanh(t), 0.3, draws)), 0.4, draws, residual=t), h)
    return L.dropout(h, 0.2, draws)


def leaf(device):
    return torch.randn(9, 40, generator=torch.Generator().manual_seed(1)).to(device).requires_grad_()


def test_a_checkpoint_draws_the_same_masks_again(device):
    x, draws = leaf(device), L.Draws(5, device)
    for step in range(3):                                   # the counter goes on from step to step
        want_out = model(x, draws, lambda f, h: f(h))
        want, = torch.autograd.grad(want_out.square().sum(), [x])
        assert draws.calls == 6
        draws.calls = 0
        out = model(x, draws, lambda f, h: checkpoint(f, h, use_reentrant=False, context_fn=draws.checkpoint))
        got, = torch.autograd.grad(out.square().sum(), [x])
        assert draws.calls == 6 and torch.equal(out, want_out) and torch.equal(got, want)
        draws.advance()
    # kept for two backward passes, and one checkpoint in another
    out = model(x, draws, lambda f, h: checkpoint(f, h, use_reentrant=False, context_fn=draws.checkpoint))
    loss = out.square().sum()
    first, = torch.autograd.grad(loss, [x], retain_graph=True)
    second, = torch.autograd.grad(loss, [x])
    assert torch.equal(first, second)
    draws.calls = 0

    def outer(t):
        return model(t, draws, lambda f, h: checkpoint(f, h, use_reentrant=False, context_fn=draws.checkpoint))

    out = checkpoint(outer, x, use_reentrant=False, context_fn=draws.checkpoint)
    nested, = torch.autograd.grad(out.square().sum(), [x])
    assert torch.equal(nested, first) and draws.calls == 6


@pytest.mark.parametrize("reentrant", [False, True])
def test_a_checkpoint_that_would_draw_others_is_refused(device, reentrant):
    x, draws = leaf(device), L.Draws(5, device)
    out = model(x, draws, lambda f, h: checkpoint(f, h, use_reentrant=reentrant))
    with pytest.raises(RuntimeError, match="other masks"):
        out.sum().backward()
    assert L.Draws(5, device).take() == 0 and draws.take() == 6                 # outside a backward pass as ever


def test_a_counter_that_was_advanced_before_it_is_refused(device):
    x, draws = leaf(device), L.Draws(5, device)
    out = checkpoint(lambda t: torch.sin(L.dropout(t, 0.5, draws)), x, use_reentrant=False, context_fn=draws.checkpoint)
    draws.advance()
    with pytest.raises(RuntimeError, match="advanced"):
        out.sum().backward()
