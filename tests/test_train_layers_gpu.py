"""The layers around a product: their gradients against 64 bits, one run of them together, graphs, streams, refusals."""

import importlib.util
import os

import pytest
import torch

import train_reference as R
from paper_2608_20818_b200 import binding as B
from paper_2608_20818_b200 import layers as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 1e-6


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def rel(got, want):
    return float(((got.double() - want).norm() / want.norm()).detach())


def mask(rows, cols, p, draws, offset):
    return R.keep(rows, cols, p, draws.seed, offset + int(draws.counter)).cuda().double() / (1 - p)


def norm64(v, w, b):
    mean = v.mean(-1, keepdim=True)
    return (v - mean) / torch.sqrt((v - mean).square().mean(-1, keepdim=True) + EPS) * w + b


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("p,with_residual,groups,add_one", [(0.0, True, 1, False), (0.2, True, 1, False), (0.2, False, 1, True),
                                                            (0.0, False, 6, True), (0.5, True, 3, True)])
def test_layer_norm_gradients(io, p, with_residual, groups, add_one):
    x, r = (randn(k, 6, 35, 200).to(io).requires_grad_() for k in (1, 2))
    w, b = ((1 + 0.2 * randn(k, *([200] if groups == 1 else [groups, 200]))).to(io).requires_grad_() for k in (3, 4))
    gy, gh = (randn(k, 6, 35, 200).to(io) for k in (5, 6))
    draws = L.Draws(77)
    draws.counter += 12345
    y, h = L.layer_norm(x, w, b, EPS, residual=r if with_residual else None, p=p, draws=draws, add_one=add_one)
    leaves = [x, w, b] + ([r] if with_residual else [])
    kept = with_residual or p > 0
    assert kept or h is x
    got = torch.autograd.grad([y, h] if kept else y, leaves, [gy, gh] if kept else gy)
    d = [t.detach().double().requires_grad_() for t in leaves]
    hd = d[0].reshape(210, 200) * (mask(210, 200, p, draws, 0) if p else 1)
    if with_residual:
        hd = hd + d[3].reshape(210, 200)
    wd, bd = (t.reshape(-1, 200).repeat_interleave(210 // groups, 0) for t in d[1:3])
    yd = norm64(hd, wd + 1 if add_one else wd, bd)
    outs = [yd.reshape(x.shape)] + ([hd.reshape(x.shape)] if kept else [])
    want = torch.autograd.grad(outs, d, [gy.double(), gh.double()][:len(outs)])
    # h is rounded (half a step of its type at most), and so is each result; the norm's gradient passes h's rounding on
    # through its three terms, each no larger than g
    room = 5 * R.store(io) if io == torch.bfloat16 else 1e-5
    assert rel(y, outs[0]) < room
    for a, e, t in zip(got, want, leaves):
        assert a.dtype == t.dtype and a.shape == t.shape and rel(a, e) < room


@pytest.mark.gpu
def test_dropout_gradients_and_both_branches_of_one_tensor():
    x, r = (randn(k, 5, 7, 130).requires_grad_() for k in (1, 2))
    g = randn(3, 5, 7, 130)
    draws = L.Draws(5)
    m = mask(35, 130, 0.3, draws, 0).reshape(x.shape)
    out = L.dropout(x, 0.3, draws, residual=r)
    assert rel(out, x.double() * m + r.double()) < 4 * R.F32
    gx, gr = torch.autograd.grad(out, [x, r], g)
    assert torch.equal(gr, g) and rel(gx, g.double() * m) < 4 * R.F32
    # x on both sides of the addition, and accumulated twice
    y, h = L.layer_norm(x, residual=x)
    (y.sum() * 0 + (h * g).sum()).backward()
    first = x.grad.clone()
    assert rel(first, 2 * g.double()) < 1e-6
    y, h = L.layer_norm(x, residual=r)
    (y * 0 + h * g).sum().backward()
    assert rel(x.grad, 3 * g.double()) < 1e-6 and rel(r.grad, g.double()) < 1e-6
    # only the stream goes on
    draws = L.Draws(6)
    _, h = L.layer_norm(x, residual=r, p=0.3, draws=draws)
    gx, gr = torch.autograd.grad(h, [x, r], g)
    assert torch.equal(gr, g) and rel(gx, g.double() * mask(35, 130, 0.3, draws, 0).reshape(x.shape)) < 4 * R.F32


@pytest.mark.gpu
@pytest.mark.parametrize("tied", [False, True])
def test_run_of_all_together(tied):
    """norm, product, dropout at the addition, norm, loss: one training step's gradients against 64 bits.  Every value that
    is kept in bf16 is off by 2^-8 / sqrt(3) of itself at most in the root of the mean square; eight such roundings lie on the
    longest way from a leaf to its gradient and back."""
    n, d, vocab, p = 320, 192, 1111, 0.1
    bf = torch.bfloat16
    x = randn(1, n, d).to(bf).requires_grad_()
    W = (randn(2, d, d) * d ** -0.5).to(bf).requires_grad_()
    E = (randn(3, vocab, d) * d ** -0.5).to(bf).requires_grad_() if tied else (randn(3, d, vocab) * d ** -0.5).to(bf).requires_grad_()
    w1, b1, w2, b2 = ((1.0 * (k % 2) + 0.1 * randn(10 + k, d)).requires_grad_() for k in (1, 2, 3, 4))
    labels = torch.randint(0, vocab, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    labels[::9] = -1
    draws = L.Draws(99)

    def step():
        y, h = L.layer_norm(x, w1, b1, EPS)
        y, h = L.layer_norm(y @ W, w2, b2, EPS, residual=h, p=p, draws=draws)
        return L.head_loss(y, E.t() if tied else E, labels).sum() / (labels >= 0).sum()

    leaves = [x, W, E, w1, b1, w2, b2]
    loss = step()
    got = torch.autograd.grad(loss, leaves)
    t = [v.detach().double().requires_grad_() for v in leaves]
    y = norm64(t[0], t[3], t[4])
    h = (y @ t[1]) * mask(n, d, p, draws, 0) + t[0]
    logits = norm64(h, t[5], t[6]) @ (t[2].t() if tied else t[2])
    live = labels >= 0
    want_loss = (torch.logsumexp(logits, 1) - logits.gather(1, labels.clamp(min=0)[:, None])[:, 0])[live].sum() / live.sum()
    want = torch.autograd.grad(want_loss, t)
    assert abs(float(loss.detach()) - float(want_loss.detach())) < 8 * R.BF16 / 3 ** 0.5 * float(want_loss.detach())
    for a, e, v in zip(got, want, leaves):
        assert a.shape == v.shape and a.dtype == v.dtype and rel(a, e) < 8 * R.BF16 / 3 ** 0.5
    # against differences: the loss along its own gradient, in the fp32 leaves (a step of 1/100 of the weights' size)
    g = got[5]
    step_size = 0.01 / float(g.norm()) * d ** 0.5
    with torch.no_grad():
        draws.calls = 0
        w2 += step_size * g
        up = float(step())
        draws.calls = 0
        w2 -= 2 * step_size * g
        down = float(step())
        w2 += step_size * g
    slope = float(g.double().square().sum()) * 2 * step_size
    # two losses, each off by the roundings' share of a mean over n rows, and the third derivative's term
    assert abs((up - down) - slope) < 0.1 * abs(slope) + 2 * R.BF16 * abs(float(loss.detach())) / n ** 0.5


@pytest.mark.gpu
def test_a_captured_step_draws_anew_at_each_replay():
    n, d, vocab, p = 96, 256, 700, 0.3
    x = randn(1, n, d).to(torch.bfloat16).requires_grad_()
    W = (randn(2, d, vocab) * d ** -0.5).to(torch.bfloat16).requires_grad_()
    w = torch.ones(d, device="cuda", requires_grad=True)
    labels = torch.randint(0, vocab, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    draws = L.Draws(31)

    def step():
        y, h = L.layer_norm(x, w, None, EPS, residual=x, p=p, draws=draws)
        y = L.dropout(y, p, draws, residual=h)
        grads = torch.autograd.grad(L.head_loss(y, W, labels).mean(), [x, W, w])
        draws.advance()
        return [y.detach(), *grads]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    draws.counter.zero_()
    eager = [step() for _ in range(3)]
    draws.counter.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    draws.counter.zero_()
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert not torch.equal(eager[0][0], eager[1][0])
    # another graph of its own, replayed on another stream beside it: no workspace is shared
    second = torch.cuda.CUDAGraph()
    with torch.cuda.graph(second):
        loss, lse = B.prm_head_loss(x.detach(), W.detach(), labels)
        gx, gw = B.prm_head_loss_backward(torch.ones(n, device="cuda"), x.detach(), W.detach(), labels, lse)
    want = [B.prm_head_loss(x.detach(), W.detach(), labels)[0], *B.prm_head_loss_backward(torch.ones(n, device="cuda"), x.detach(), W.detach(), labels, B.prm_head_loss(x.detach(), W.detach(), labels)[1])]
    torch.cuda.synchronize()
    for _ in range(5):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            second.replay()
        graph.replay()
        torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(loss, want[0]) and torch.equal(gx, want[1]) and torch.equal(gw, want[2])


@pytest.mark.gpu
def test_calls_on_another_stream():
    x, r = (randn(k, 300, 512) for k in (1, 2))
    w = torch.ones(512, device="cuda")
    xb, W = randn(3, 40, 64).to(torch.bfloat16), randn(4, 64, 900).to(torch.bfloat16)
    labels, gl = torch.arange(40, device="cuda"), torch.ones(40, device="cuda")

    def all_of(stream):
        y, h, mean, rstd = B.prm_layernorm(x, w, w, EPS, residual=r, p=0.2, seed=1, stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
            stream.wait_stream(torch.cuda.current_stream())
        out = [y, h, *B.prm_layernorm_backward(y, h, mean, rstd, w, p=0.2, seed=1, stream=stream)]
        out.append(B.prm_dropout(x, 0.2, 1, residual=r, stream=stream))
        loss, lse = B.prm_head_loss(xb, W, labels, stream=stream)
        out += [loss, *B.prm_head_loss_backward(gl, xb, W, labels, lse, stream=stream)]
        return out

    want = all_of(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = all_of(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_layer_refusals():
    x = randn(1, 6, 64).requires_grad_()
    draws = L.Draws(1)
    for f in (lambda: L.dropout(x, 0.5, None), lambda: L.dropout(x, 0.5, draws, residual=x[:3]), lambda: L.layer_norm(x, residual=x[:3]),
              lambda: L.layer_norm(x, p=0.5), lambda: L.dropout(x, 1.0, draws),
              lambda: L.head_loss(x.bfloat16(), randn(2, 64, 9).bfloat16(), torch.zeros(5, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    out = L.dropout(x, 0.5, draws)
    draws.advance()                              # before the backward pass: another mask
    with pytest.raises(RuntimeError):
        out.sum().backward()
    xb, W = x.detach().bfloat16().requires_grad_(), randn(2, 64, 9).bfloat16().requires_grad_()
    labels = torch.zeros(6, dtype=torch.int64, device="cuda")
    # another path keeps the graph of a second derivative alive beside the layer
    for f, leaf in ((lambda: L.dropout(x, 0.5, draws).square().sum() + x.pow(3).sum(), x),
                    (lambda: L.layer_norm(x)[0].square().sum() + x.pow(3).sum(), x),
                    (lambda: L.head_loss(xb, W, labels).sum() + xb.pow(3).sum(), xb)):
        with pytest.raises(RuntimeError):
            torch.autograd.grad(f(), [leaf], create_graph=True)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_example_runs(fmt):
    spec = importlib.util.spec_from_file_location("train_tokens_q8", os.path.join(ROOT, "examples", "train_tokens_q8.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(steps=4, vocab=301, dim=128, blocks=2, tokens=500, format=fmt, log=None)
    assert len(losses) == 4 and all(v == v and abs(v) < 100 for v in losses)
