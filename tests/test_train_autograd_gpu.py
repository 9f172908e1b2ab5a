"""What autograd allows of any function's results, and the layers' have to allow too."""

import pytest
import torch

from paper_2608_20818_b200 import layers as L


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def dropped(x, w, draws):
    return L.dropout(x, 0.4, draws)


def added(x, w, draws):
    return L.dropout(x, 0.4, draws, residual=x)


def normed(x, w, draws):
    return L.layer_norm(x, w)[0]


def normed_sum(x, w, draws):
    return L.layer_norm(x, w, residual=x, p=0.3, draws=draws)[0]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(6, 72), (2, 3, 72), (72,)])
@pytest.mark.parametrize("f", [dropped, added, normed, normed_sum])
def test_results_may_be_written_to(f, shape):
    """In place, it is the same calculation; the stream h, which the gradient reads, is refused by autograd itself."""
    x, w, g = randn(1, *shape).requires_grad_(), randn(2, 72).requires_grad_(), randn(3, *shape)
    want = torch.autograd.grad(torch.relu(f(x, w, L.Draws(3)) * 2), [x, w], g, allow_unused=True)
    y = f(x, w, L.Draws(3))
    got = torch.autograd.grad(y.mul_(2).relu_(), [x, w], g, allow_unused=True)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, want))
    y, h = L.layer_norm(x, w, residual=x)
    h.add_(1)
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(5, 0), (2, 0, 72), (0,), (0, 72)])
def test_nothing_is_dropped_out_of_nothing(shape):
    x = randn(1, *shape).requires_grad_()
    for residual in (None, x):
        out = L.dropout(x, 0.5, L.Draws(1), residual=residual)
        grad, = torch.autograd.grad(out.sum(), [x])
        assert out.shape == grad.shape == x.shape
    if shape[-1]:
        y, h = L.layer_norm(x, torch.ones(shape[-1], device="cuda"), residual=x, p=0.5, draws=L.Draws(1))
        grad, = torch.autograd.grad((y + h).sum(), [x])
        assert y.shape == h.shape == grad.shape == x.shape
