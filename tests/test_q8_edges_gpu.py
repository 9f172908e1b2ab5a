"""Edges of the 8-bit operators: the documented rounding bit by bit, sizes and values at the ends of their ranges."""

import os
import subprocess
import sys

import pytest
import torch

import q8_reference as R
from paper_2608_20818_b200 import binding as B
from paper_2608_20818_b200 import q8 as Q

EPS = 1e-6


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def codes_by_the_rule(t, dim, fmt):
    """round(t * (limit * (1 / T))) with each step rounded to fp32, on the host."""
    t = t.cpu()
    v = t * (R.LIMIT[fmt] * (1.0 / t.abs().amax(dim, keepdim=True)))
    return (v.round() if fmt == "int8" else v).to(R.EIGHT[fmt]).float()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
# rows in registers, rows that start anywhere, single elements; columns by panels, streamed (one and two rows
# per set), and single elements
@pytest.mark.parametrize("rows,cols", [(700, 256), (90, 2048), (160, 1111), (5, 40001), (900, 515), (4200, 4096),
                                       (8300, 512), (2100, 9000)])
def test_codes_follow_the_rule_bit_by_bit(rows, cols, io, fmt):
    x = randn(rows + cols, rows, cols).to(io)
    w = (1 + 0.2 * randn(cols, cols)).to(io)
    fr, fc = torch.exp(randn(rows, rows)), torch.exp(randn(cols + 1, cols))
    q, _, _ = B.prm_rmsnorm_q8(x, w, EPS, format=fmt)
    assert torch.equal(q.float().cpu(), codes_by_the_rule(x.float() * w.float(), 1, fmt))
    qr, _, qc, _ = B.prm_quantize_q8(x, by_cols=True, fold_rows=fr, fold_cols=fc, format=fmt)
    assert torch.equal(qr.float().cpu(), codes_by_the_rule(x.float() * fc, 1, fmt))
    assert torch.equal(qc.float().cpu(), codes_by_the_rule(x.float() * fr[:, None], 0, fmt))


def check_norm_backward(gy, h, w, eps, gh):
    gx, gw = B.prm_rmsnorm_q8_backward(gy, h, w, eps, grad_h=gh)
    rx, rw, sx, sw = R.norm_backward(gy, h, w, eps, gh)
    # every term goes through the two row sums and a handful of products, 100 roundings at most; grad_w is added
    # over the rows in turn at worst
    for got, ref, size, rounds in ((gx, rx, sx, 100), (gw, rw, sw, 100 + len(h))):
        store = R.BF16 if got.dtype == torch.bfloat16 else R.F32
        assert torch.all((got.double() - ref).abs() <= rounds * R.F32 * size + 1.01 * store * ref.abs())


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
# wide rows of odd widths, more of them than blocks
@pytest.mark.parametrize("rows,cols", [(149, 6139), (310, 8185), (160, 8187), (300, 9001), (160, 16377), (1500, 6141)])
def test_norm_backward_of_many_wide_odd_rows(rows, cols, io):
    h, gy, gh = (randn(rows + cols + k, rows, cols).to(io) for k in range(3))
    w = (1 + 0.2 * randn(cols, cols)).to(io)
    check_norm_backward(gy, h, w, EPS, gh)
    check_norm_backward(gy, h, w, EPS, None)


@pytest.mark.gpu
def test_second_derivatives_are_refused():
    """Other paths (the residual stream, a term of the weight) keep the graph of a second derivative alive beside
    the layers: their terms must not drop out of it silently."""
    x, r = (randn(k, 6, 64).requires_grad_() for k in (1, 2))
    n = torch.ones(64, device="cuda", requires_grad=True)
    W = randn(3, 64, 32).requires_grad_()
    w8 = Q.Weight8(W)
    for f in (lambda: Q.norm_linear(x, r, n, w8)[0].square().sum() + x.pow(3).sum(),
              lambda: Q.norm_linear(x, None, n, w8)[0].sum() + x.pow(3).sum(),
              lambda: Q.linear(x, w8).square().sum() + x.pow(3).sum(),
              lambda: Q.linear(x, w8).sum() + W.pow(3).sum() + x.pow(3).sum()):
        first = torch.autograd.grad(f(), [x, W], allow_unused=True)
        assert all(g is not None for g in first)
        with pytest.raises(RuntimeError):
            gx, gw = torch.autograd.grad(f(), [x, W], create_graph=True)
            torch.autograd.grad(gx.square().sum() + gw.square().sum(), x)


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [(), (1,), (2, 3), (2, 0), (0,)])
def test_layers_take_any_leading_dimensions(lead):
    """One vector, no tokens at all: as the rows of a matrix, gradients too."""
    W, n = randn(3, 64, 32).requires_grad_(), torch.ones(64, device="cuda", requires_grad=True)
    w8 = Q.Weight8(W)
    x, r = (randn(k, *lead, 64).requires_grad_() for k in (1, 2))
    gy, gh = randn(4, *lead, 32), randn(5, *lead, 64)

    def run(f, x, r, gy, gh):
        y, h = f(x, r)
        return y, h, torch.autograd.grad([y, h], [x, r, n, W], [gy, gh])

    flat = lambda t: t.detach().reshape(-1, t.shape[-1])  # noqa: E731
    for f in (lambda x, r: Q.norm_linear(x, r, n, w8),
              lambda x, r: (Q.norm_linear(x, None, n, w8)[0], x + r),
              lambda x, r: (Q.linear(x, w8) + n.sum(), x + r)):
        y, h, got = run(f, x, r, gy, gh)
        assert y.shape == (*lead, 32) and h.shape == (*lead, 64)
        y2, h2, want = run(f, flat(x).requires_grad_(), flat(r).requires_grad_(), flat(gy), flat(gh))
        assert torch.equal(flat(y), y2) and torch.equal(flat(h), h2)
        assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip(got, want))
        assert [g.shape for g in got] == [t.shape for t in (x, r, n, W)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(6, 64), (2, 3, 64)])
def test_gradients_of_x_and_residual_accumulate_apart(shape):
    """Both get the same gradient; what is added to one in a later backward pass must not reach the other."""
    n = torch.ones(64, device="cuda", requires_grad=True)
    w8 = Q.Weight8(randn(3, 64, 32).requires_grad_())
    gy, gh = randn(4, *shape[:-1], 32), randn(5, *shape)
    for used in ((0, 1), (0,), (1,)):
        x, r = (randn(k, *shape).requires_grad_() for k in (1, 2))

        def out():
            both = Q.norm_linear(x, r, n, w8)
            return [both[i] for i in used], [(gy, gh)[i] for i in used]

        one, = torch.autograd.grad(out()[0], x, out()[1])
        for _ in range(3):
            torch.autograd.backward(*out())
        assert torch.equal(x.grad, one + one + one) and torch.equal(r.grad, x.grad)
        assert x.grad.data_ptr() != r.grad.data_ptr()


STALE_ERROR = """
import torch
from paper_2608_20818_b200 import binding as B

opt = B.PeriodicRowwiseMuon([(64, 64)], K=5, beta=0.9, nesterov=True, lr=0.1, wd=0.0)
weight, grad = (torch.ones(64, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
momentum = torch.zeros(64, 64, device="cuda")
opt.step([weight], [grad], [momentum], 1)
x = torch.randn(300, 256, device="cuda")
w = torch.ones(256, device="cuda")
torch.cuda.synchronize()


def during_capture(call):
    # A stream under capture cannot be waited for: CUDA refuses on the host, and the error stays the thread's last.
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        code = call()
        try:
            graph.capture_end()
        except RuntimeError:
            pass
    return code


calls = [lambda: B.prm_rmsnorm_q8(x, w, 1e-6), lambda: B.prm_rmsnorm_q8(x[:, :255], w[:255], 1e-6),
         lambda: B.prm_quantize_q8(x), lambda: B.prm_quantize_q8(x[:, :255]), lambda: B.prm_quantize_q8(x, by_cols=True),
         lambda: B.prm_quantize_q8(x[:, :255], by_rows=False, by_cols=True), lambda: B.prm_rmsnorm_q8_backward(x, x, w, 1e-6)]
for call in calls:
    assert during_capture(lambda: B.prm_status(opt.h)) == B.PRM_ERR_CUDA
    call()
assert during_capture(B.prm_q8_status) == B.PRM_ERR_CUDA       # leaves no error for the next to find
B.prm_adamw_step([w], [torch.ones_like(w)], [torch.zeros_like(w)], [torch.zeros_like(w)], 1, lr=1e-3)
torch.cuda.synchronize()
print("done")
"""


@pytest.mark.gpu
def test_errors_of_other_calls_are_not_theirs():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", STALE_ERROR], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.stdout.strip() == "done", run.stderr[-2000:]


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
# each of the gradient's kernels: groups, wide, streamed, rows that start anywhere, single elements
@pytest.mark.parametrize("rows,cols", [(6, 64), (5, 2048), (4, 6000), (400, 6000), (7, 515), (3, 16384)])
def test_norm_backward_of_large_and_small_rows(rows, cols, io):
    """Rows of root mean squares from 1e-15 to 1e15: the powers of s stay in range where the gradient does."""
    size = torch.tensor([1e-15, 1e15, 1.0, 1e-13, 1e13], device="cuda")[torch.arange(rows, device="cuda") % 5, None]
    h, gy, gh = ((randn(rows + cols + k, rows, cols) * s).to(io) for k, s in enumerate((size, 1, 0.01 / size)))
    check_norm_backward(gy, h, (1 + 0.2 * randn(cols, cols)).to(io), 0.0, gh)
    check_norm_backward(gy, h, (1 + 0.2 * randn(cols, cols)).to(io), 0.0, None)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("cols", [64, 515, 2048, 40001])
def test_zero_rows_without_eps(cols, fmt):
    x = randn(cols, 4, cols)
    x[1] = 0
    x[2] = 2.0 ** -110
    for r in (None, torch.zeros_like(x)):
        q, scale, _ = B.prm_rmsnorm_q8(x, torch.ones(cols, device="cuda"), 0.0, residual=r, format=fmt)
        assert not q[1:3].float().any() and not scale[1:3].any() and torch.all(scale[[0, 3]] > 0)
