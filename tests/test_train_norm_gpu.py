"""Layer norm and its gradient where rows are constant, far from zero or no numbers, in all layouts, against 64 bits."""

import pytest
import torch

import train_reference as R
from paper_2608_20818_b200 import binding as B

# columns, and how the stream lies: aligned, starting anywhere, starting unlike its gradient (single elements), too wide for registers
LAYOUTS = [(64, "aligned"), (200, "aligned"), (1024, "aligned"), (4096, "aligned"), (8192, "aligned"), (63, "shifted"), (1023, "shifted"),
           (4099, "shifted"), (1024, "unlike"), (12000, "wide")]
TYPES = [torch.bfloat16, torch.float32]


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def close(got, want, room, what):
    bad = (got.double() - want).abs() - room
    assert torch.all(bad <= 0), (what, float(bad.max()))


def unlike(t, how):
    """The matrix in rows that start one element off, where that is what is asked for."""
    if how != "unlike":
        return t
    wide = torch.empty(t.shape[0], t.shape[1] + 3, dtype=t.dtype, device=t.device)
    wide[:, 1:-2] = t
    return wide[:, 1:-2]


@pytest.mark.gpu
@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("cols,how", LAYOUTS)
def test_gradient_of_constant_rows(cols, how, io):
    """xhat is 0: they give the weight nothing, and grad_r is rstd (g - mean g)."""
    rows, eps = 70, 1e-5
    h = (301.0 + 7.0 * torch.arange(rows, device="cuda"))[:, None].expand(rows, cols).to(io).contiguous()
    gy, w = randn(cols, rows, cols).to(io), 1 + 0.2 * randn(1, cols)
    y, _, mean, rstd = B.prm_layernorm(h, w, None, eps)
    assert torch.all(y == 0) and torch.equal(mean, h[:, 0].float())
    gx, _, gw, gb = B.prm_layernorm_backward(unlike(gy, how), h, mean, rstd, w)
    assert torch.all(gw == 0)
    g = gy.double() * w.double()
    want = rstd.double()[:, None] * (g - g.mean(1, keepdim=True))
    size = rstd.double()[:, None] * (g.abs() + g.abs().mean(1, keepdim=True))
    # a thread adds 64 numbers in a row at most, then 10 by shuffles; a handful of products
    close(gx, want, 100 * R.F32 * size + 1.01 * R.store(io) * want.abs(), "grad_x")


@pytest.mark.gpu
@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("cols,how", LAYOUTS)
def test_gradient_of_rows_far_from_zero(cols, how, io):
    """Means of 10^4 deviations: what is off in xhat = (h - mean) rstd goes by xhat, not by the mean."""
    rows = 70
    h = (100.0 + 100.0 * torch.rand(rows, 1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) + 0.01 * randn(3, rows, cols)).to(io)
    gy, w = randn(cols, rows, cols).to(io), 1 + 0.2 * randn(1, cols)
    _, _, mean, rstd = B.prm_layernorm(h, w, None, 1e-6)
    gx, _, gw, gb = B.prm_layernorm_backward(unlike(gy, how), h, mean, rstd, w)
    r = rstd.double()[:, None]
    xhat = (h.double() - mean.double()[:, None]) * r
    g = gy.double() * w.double()
    want = r * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    size = r * (g.abs() + g.abs().mean(1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    close(gx, want, 100 * R.F32 * size + 1.01 * R.store(io) * want.abs(), "grad_x")
    rounds = 100 + rows
    for got, terms in ((gw, gy.double() * xhat), (gb, gy.double())):
        close(got, terms.sum(0), rounds * R.F32 * terms.abs().sum(0) + 1.01 * R.F32 * terms.sum(0).abs(), "grad_w, grad_b")

@pytest.mark.gpu
@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("rows,cols,how", [(40, c, h) for c, h in LAYOUTS] + [(9000, 1100, "aligned"), (5001, 2001, "shifted"), (3000, 4096, "aligned")])
def test_forward_of_rows_far_from_zero(rows, cols, how, io):
    """y goes by h - mean: the mean that the row was reduced with is off by its own rounding and that of the sums, which the second
    reduction takes off again.  What is left is the rounding of the sum of h - (first mean), and a few steps of y."""
    h = (100.0 + 100.0 * torch.rand(rows, 1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) + 0.01 * randn(3, rows, cols)).to(io)
    w, b = 1 + 0.2 * randn(1, cols), randn(4, cols)
    y, _, mean, rstd = B.prm_layernorm(unlike(h, how), w, b, 1e-6)
    v = h.double()
    m = v.mean(1, keepdim=True)
    rs = 1 / torch.sqrt((v - m).square().mean(1, keepdim=True) + 1e-6)
    # first mean: 80 sums of which each is off by half a step of the row's mean at most
    first = 80 * R.F32 * m.abs()
    off = 100 * R.F32 * ((v - m).abs().mean(1, keepdim=True) + first) + R.F32 * ((v - m).abs() + first)
    # the variance is sums of squares of h - first, less the square of what is taken off
    spread = 100 * R.F32 * ((v - m).square().mean(1, keepdim=True) + 2 * first.square()) * rs.square()
    want = (v - m) * rs * w.double() + b.double()
    size = ((v - m).abs() + off) * rs * w.double().abs()
    room = off * rs * w.double().abs() + size * (spread + 8 * R.F32) + 2 * R.F32 * (size + b.double().abs())
    close(y, want, room + 1.01 * R.store(io) * want.abs(), "y")
    assert io != torch.float32 or float(room.max()) < 0.05          # the bound says something: y itself is about 1
    close(rstd, rs[:, 0], (rs * (spread + 4 * R.F32))[:, 0], "rstd")


@pytest.mark.gpu
@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("rows,cols,how", [(70, c, h) for c, h in LAYOUTS] + [(9000, 1100, "aligned"), (5001, 2001, "shifted"), (3000, 4096, "aligned")])
def test_statistics_of_rows_that_are_no_numbers(rows, cols, how, io):
    """What the formulas give: a NaN leaves mean and rstd NaN, an infinity an infinite mean and rstd NaN; squares beyond fp32 leave
    rstd 0 and y = bias.  No other row is touched."""
    h, b = randn(cols, rows, cols).to(io), randn(4, cols)
    y0, _, mean0, rstd0 = B.prm_layernorm(unlike(h, how), None, b)
    h[3, cols // 2] = float("nan")
    h[5, 0] = float("inf")
    h[rows - 2, cols - 1] = float("-inf")
    h[9] = torch.where(torch.arange(cols, device="cuda") % 2 == 0, 1e30, -1e30).to(io)
    h[10] = 1e34
    y, _, mean, rstd = B.prm_layernorm(unlike(h, how), None, b)
    odd = [3, 5, rows - 2]
    assert bool(torch.isnan(mean[3])) and float(mean[5]) == float("inf") and float(mean[rows - 2]) == float("-inf")
    assert torch.all(torch.isnan(rstd[odd])) and torch.all(torch.isnan(y[odd]))
    assert float(rstd[9]) == 0 and torch.equal(y[9], b.to(io)) and torch.equal(y[10], b.to(io))
    rest = [i for i in range(rows) if i not in odd + [9, 10]]
    assert torch.equal(y[rest], y0[rest]) and torch.equal(mean[rest], mean0[rest]) and torch.equal(rstd[rest], rstd0[rest])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,per,cols", [(4000000, 1, 8), (4000000, 2, 9), (2000001, 1, 40)])
def test_gradient_of_millions_of_groups(rows, per, cols):
    """A weight for each row or two: what the forward pass takes, its gradient takes too."""
    groups = rows // per
    h, gy = randn(1, rows, cols), randn(2, rows, cols)
    w = 1 + 0.2 * randn(3, groups, cols)
    y, _, mean, rstd = B.prm_layernorm(h, w, w)
    gx, _, gw, gb = B.prm_layernorm_backward(gy, h, mean, rstd, w)
    rx, rw, rb, sx, sw, sb = R.norm_backward(gy, h, mean, rstd, w)
    close(gx, rx, 100 * R.F32 * sx + 1.01 * R.F32 * rx.abs(), "grad_x")
    close(gw, rw, 100 * R.F32 * sw + 1.01 * R.F32 * rw.abs(), "grad_w")
    close(gb, rb, 100 * R.F32 * sb + 1.01 * R.F32 * rb.abs(), "grad_b")


@pytest.mark.gpu
@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("groups,per,cols", [(300, 20, 1024), (1024, 8, 512), (200, 9, 200), (149, 33, 2048)])
@pytest.mark.parametrize("start,ld", [(0, 0), (8, 8), (3, 8), (1, 3)])
def test_gradient_of_many_groups_in_any_rows(groups, per, cols, start, ld, io):
    """Whole octs, aligned or not, in rows that start alike (a stride of octs) or do not: no more scratch than there is is written."""
    rows = groups * per

    def place(t=None):
        wide = torch.full((rows, cols + ld + 8), float("nan"), dtype=io, device="cuda")[:, :cols + ld]
        wide = wide.as_strided((rows, cols), (cols + ld, 1), start)
        return wide if t is None else wide.copy_(t)

    h, gy = place(randn(1, rows, cols)), place(randn(2, rows, cols))
    w = 1 + 0.2 * randn(3, groups, cols)
    _, _, mean, rstd = B.prm_layernorm(h, w)
    gr, gw, gb = place(), torch.empty_like(w), torch.empty_like(w)
    nbytes = B.lib().prm_layernorm_scratch_bytes(rows, cols, per)
    scratch = torch.full((nbytes + 4096,), 77, dtype=torch.uint8, device="cuda")
    code = B.lib().prm_layernorm_backward(gy.data_ptr(), cols + ld, h.data_ptr(), cols + ld, mean.data_ptr(), rstd.data_ptr(), w.data_ptr(),
                                          cols, None, 0, rows, cols, per, int(io == torch.float32), 1, 0, 0.0, 0, 0, None, gr.data_ptr(),
                                          cols + ld, None, 0, gw.data_ptr(), gb.data_ptr(), scratch.data_ptr(), nbytes,
                                          torch.cuda.current_stream().cuda_stream)
    assert code == B.PRM_OK
    rx, rw, rb, sx, sw, sb = R.norm_backward(gy, h, mean, rstd, w)
    close(gr, rx, 100 * R.F32 * sx + 1.01 * R.store(io) * rx.abs(), "grad_r")
    close(gw, rw, (100 + per) * R.F32 * sw + 1.01 * R.F32 * rw.abs(), "grad_w")
    close(gb, rb, (100 + per) * R.F32 * sb + 1.01 * R.F32 * rb.abs(), "grad_b")
    assert torch.all(scratch[nbytes:] == 77)
