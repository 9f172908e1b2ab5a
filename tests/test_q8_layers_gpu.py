"""8-bit linear layers: their gradients against the formulas on the quantised values, and a short training
run with the optimizer."""

import importlib.util
import os

import pytest
import torch

import q8_reference as R
from paper_2608_20818_b200 import q8 as Q

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 1e-6


def rel(got, want):
    return float(((got.double() - want).norm() / want.norm()).detach())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("with_residual", [True, False])
def test_norm_linear_and_gradients(fmt, dtype, with_residual):
    """Against the same layer in 64 bits without any rounding to 8 bits.  A value of 8 bits is off by at most
    half a step: 1/254 of its row's largest magnitude in int8 (rms 1/254/sqrt(3) of it, the largest being
    about 4 times the row's rms), 2^-4 of itself in e4m3 (rms about 2^-4/sqrt(3)); both operands of each of
    the products, the second of them after the norm's gradient, add in squares."""
    one = 4 / 254 / 3 ** 0.5 if fmt == "int8" else 2.0 ** -4 / 3 ** 0.5
    g = torch.Generator(device="cuda").manual_seed(3)
    x, r = (torch.randn(3, 70, 256, generator=g, device="cuda").to(dtype).requires_grad_() for _ in range(2))
    n = (1 + 0.1 * torch.randn(256, generator=g, device="cuda")).requires_grad_()
    W = (torch.randn(256, 384, generator=g, device="cuda") / 16).to(dtype).requires_grad_()
    gy = torch.randn(3, 70, 384, generator=g, device="cuda").to(dtype)
    gh = torch.randn(3, 70, 256, generator=g, device="cuda").to(dtype)
    w8 = Q.Weight8(W, fmt)
    y, h = Q.norm_linear(x, r if with_residual else None, n, w8, EPS)
    leaves = [x, n, W] + ([r] if with_residual else [])
    got = torch.autograd.grad([y, h], leaves, [gy, gh]) if with_residual else torch.autograd.grad(y, leaves, gy)
    d = [t.detach().double().requires_grad_() for t in leaves]
    hd = d[0] + d[3] if with_residual else d[0]
    yd = R.norm_output(hd.reshape(-1, 256), d[1], EPS).reshape(hd.shape) @ d[2]
    want = torch.autograd.grad([yd, hd], d, [gy.double(), gh.double()]) if with_residual else torch.autograd.grad(yd, d, gy.double())
    assert y.dtype == dtype and rel(y, yd) < 2 * one
    for a, b, t in zip(got, want, leaves):
        assert a.dtype == t.dtype and a.shape == t.shape and rel(a, b) < 3 * one
    assert not with_residual or torch.equal(got[0], got[3])


@pytest.mark.gpu
def test_linear_gradients_are_exact_products_of_the_codes():
    """Given the codes, the two gradients are the products that they stand for, rounded once."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(33, 130, generator=g, device="cuda").requires_grad_()
    W = torch.randn(130, 77, generator=g, device="cuda").requires_grad_()
    gy = torch.randn(33, 77, generator=g, device="cuda")
    w8 = Q.Weight8(W)
    Q.linear(x, w8).backward(gy)
    x8, sx, _, _ = Q.prm_quantize_q8(x.detach())
    gr, sr, gc, sc = Q.prm_quantize_q8(gy, by_cols=True, fold_rows=sx, fold_cols=w8.scale)
    for got, ref in ((x.grad, R.matmul(gr, sr, w8.codes.t(), None)), (W.grad, R.matmul(x8.t(), None, gc, sc))):
        assert torch.all((got.double() - ref).abs() <= 4 * R.F32 * ref.abs())


@pytest.mark.gpu
def test_what_needs_no_gradient():
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(5, 64, generator=g, device="cuda")
    W = torch.randn(64, 32, generator=g, device="cuda").requires_grad_()
    n = torch.ones(64, device="cuda")
    w8 = Q.Weight8(W)
    Q.linear(x, w8).sum().backward()
    first = W.grad.clone()
    Q.norm_linear(x, x, n, w8)[0].sum().backward()
    assert first.abs().sum() > 0 and not torch.equal(W.grad, first)
    x.requires_grad_()
    Q.norm_linear(x, x.detach(), n, w8)[1].sum().backward()      # only the stream is used
    assert torch.all(x.grad == 1)
    with pytest.raises(ValueError):
        Q.norm_linear(x, x[:2], n, w8)


@pytest.mark.gpu
def test_layers_train_with_the_optimizer():
    """The example's short run: in either format the loss falls as it does with bf16 layers."""
    spec = importlib.util.spec_from_file_location("train_mlp_q8", os.path.join(ROOT, "examples", "train_mlp_q8.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = {f: example.train(steps=30, dim=256, blocks=2, tokens=1024, format=f, log=None) for f in ("bf16", "int8", "e4m3")}
    for f in ("int8", "e4m3"):
        assert losses[f][-1] < 0.7 * losses[f][0]
        assert abs(losses[f][-1] - losses["bf16"][-1]) < 0.1 * losses["bf16"][0]
