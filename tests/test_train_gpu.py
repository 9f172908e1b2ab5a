"""Dropout, layer norm and the loss of a linear head against 64-bit forms."""

import pytest
import torch

import train_reference as R
from paper_2608_20818_b200 import binding as B

EPS = 1e-6
TYPES = [torch.bfloat16, torch.float32]


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def laid(t, how):
    """The matrix stored as it is, with rows 8 elements longer, or with rows that start anywhere."""
    if how == "dense":
        return t
    rows, cols = t.shape
    wide = torch.full((rows, cols + (8 if how == "padded" else 3)), float("nan"), dtype=t.dtype, device=t.device)
    start = 0 if how == "padded" else 1
    wide[:, start:start + cols] = t
    return wide[:, start:start + cols]


def close(got, want, room, what):
    bad = (got.double() - want).abs() - room
    assert torch.all(bad <= 0), (what, float(bad.max()))


# ------------------------------------------------------------------ dropout

@pytest.mark.gpu
@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 3), (5, 8), (3, 70), (33, 256), (7, 1000), (130, 1111), (9, 8200), (2, 40001)])
@pytest.mark.parametrize("how", ["dense", "padded", "ragged"])
def test_dropout_bit_by_bit(rows, cols, io, how):
    x, r = laid(randn(rows + cols, rows, cols).to(io), how), randn(cols, rows, cols).to(io)
    counter = torch.tensor([2 ** 33 + 5], device="cuda")
    for p, seed, offset, c, res in ((0.1, 2 ** 63 + 12345, 3, counter, None), (0.5, 7, 2 ** 64 - 1, None, laid(r, how)), (0.9, -1, 0, counter, r),
                                    (0.0, 1, 0, None, r)):
        out = B.prm_dropout(x, p, seed, offset, counter=c, residual=res)
        want = R.dropped(x.float(), p, seed, offset + (int(c) if c is not None else 0))
        want = want if res is None else want + res.float()
        assert out.dtype == io and torch.equal(out, want.to(io)), (p, how)


@pytest.mark.gpu
def test_dropout_of_what_is_no_number_and_of_nothing():
    x = torch.full((64, 64), float("inf"), device="cuda")
    x[::2] = float("nan")
    out = B.prm_dropout(x, 0.5, 11)
    kept = R.keep(64, 64, 0.5, 11, 0).cuda()
    assert torch.all(out[~kept] == 0) and not torch.any(torch.isfinite(out[kept]))
    assert B.prm_dropout(x[:0], 0.5, 1).shape == (0, 64) and B.prm_dropout(x[:, :0], 0.5, 1).shape == (64, 0)


@pytest.mark.gpu
def test_a_probability_too_small_to_drop_anything():
    """Below half of 2^-32: what dropout returns is there all the same."""
    x = randn(1, 30, 200)
    y, h, _, _ = B.prm_layernorm(x, p=1e-12, seed=3)
    assert torch.equal(h, x) and torch.equal(y, B.prm_layernorm(x)[0]) and torch.equal(B.prm_dropout(x, 1e-12, 3), x)
    gx, gr, _, _ = B.prm_layernorm_backward(x, h, *B.prm_layernorm(x)[2:], p=1e-12, seed=3)
    assert torch.equal(gx, gr)


@pytest.mark.gpu
def test_dropout_beyond_32_bits_of_offsets():
    """The last rows of a matrix of more than 2^32 bytes and 2^31 elements."""
    rows, cols = 70000, 32768
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    out = B.prm_dropout(x, 0.25, 5)
    k = R.keep(rows, 8, 0.25, 5, 0)[-50:].cuda()               # a row's first words do not depend on its length
    assert torch.equal(out[-50:, :8] != 0, k)


# --------------------------------------------------------------- layer norm

def affine(rows, cols, groups, wt, seed, how="dense"):
    wide = (1 + 0.2 * randn(seed, groups, 6 * cols)).to(wt)
    w, b = wide[:, cols:2 * cols], wide[:, 3 * cols:4 * cols]
    return (w[0], b[0]) if groups == 1 else (w, b)


def check_norm(x, r, w, b, add_one, p, seed=9, offset=4, counter=None):
    y, h, mean, rstd = B.prm_layernorm(x, w, b, EPS, residual=r, add_one=add_one, p=p, seed=seed, offset=offset, counter=counter)
    want = R.dropped(x.float(), p, seed, offset + (int(counter) if counter is not None else 0))
    want = (want if r is None else want + r.float()).to(x.dtype)
    if r is None and p == 0:
        assert h is None
    else:
        assert torch.equal(h, want)
    ry, rm, rr, size = R.norm(want, w, b, EPS, add_one)
    # a thread adds 64 numbers in a row at most, then 10 by shuffles; the products and the root are a handful more
    close(mean, rm, 100 * R.F32 * want.double().abs().mean(1), "mean")
    close(rstd, rr, 200 * R.F32 * rr, "rstd")
    close(y, ry, 200 * R.F32 * size + 1.01 * R.store(x.dtype) * ry.abs(), "y")
    return want, mean, rstd


def check_norm_backward(gy, h, mean, rstd, w, gh, add_one, p, seed=9, offset=4, counter=None):
    gx, gr, gw, gb = B.prm_layernorm_backward(gy, h, mean, rstd, w, grad_h=gh, add_one=add_one, p=p, seed=seed, offset=offset,
                                              counter=counter)
    rr, rw, rb, sr, sw, sb = R.norm_backward(gy, h, mean, rstd, w, gh, add_one)
    store = R.store(h.dtype)
    if p > 0:
        close(gr, rr, 100 * R.F32 * sr + 1.01 * store * rr.abs(), "grad_residual")
        k = R.keep(*h.shape, p, seed, offset + (int(counter) if counter is not None else 0)).cuda()
        want = torch.where(k, rr / (1 - p), torch.zeros_like(rr))
        close(gx, want, (100 * R.F32 * sr + 1.01 * store * rr.abs()) / (1 - p) + R.F32 * want.abs(), "grad_x")
    else:
        assert gr is None
        close(gx, rr, 100 * R.F32 * sr + 1.01 * store * rr.abs(), "grad_x")
    rounds = 100 + len(h)                  # the rows' terms, added in turn at worst
    for got, ref, size, name in ((gw, rw, sw, "grad_w"), (gb, rb, sb, "grad_b")):
        assert got.shape == ref.shape and (w is None or got.dtype == w.dtype)
        close(got, ref, rounds * R.F32 * size + 1.01 * R.store(got.dtype) * ref.abs(), name)


SHAPES = [(1, 1), (1, 5), (3, 64), (40, 64), (17, 200), (33, 256), (5, 511), (9, 512), (30, 1000), (700, 1024), (5, 1111),
          (65, 2048), (20, 2050), (12, 4096), (11, 4100), (7, 8192), (3, 10000), (2, 16384), (2, 20001)]


@pytest.mark.gpu
@pytest.mark.parametrize("io,wt", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("how", ["dense", "padded", "ragged"])
def test_layernorm_and_gradient(rows, cols, io, wt, how):
    x, r = (laid((randn(rows * 3 + cols + k, rows, cols) + 2 * k).to(io), how) for k in range(2))
    gy, gh = ((randn(rows + cols + 7 + k, rows, cols) * 0.01).to(io) for k in range(2))
    w, b = affine(rows, cols, 1, wt, cols)
    counter = torch.tensor([2 ** 35 + 1], device="cuda")
    h, mean, rstd = check_norm(x, r, w, b, False, 0.0)
    check_norm_backward(laid(gy, how), laid(h, how), mean, rstd, w, laid(gh, how), False, 0.0)
    h, mean, rstd = check_norm(x, r, w, b, True, 0.25, counter=counter)
    check_norm_backward(gy, h, mean, rstd, w, gh, True, 0.25, counter=counter)
    h, mean, rstd = check_norm(x, None, w, b, False, 0.0)
    check_norm_backward(gy, x, mean, rstd, w, None, False, 0.0)
    h, mean, rstd = check_norm(x, None, None, None, False, 0.5)
    check_norm_backward(laid(gy, how), h, mean, rstd, None, None, False, 0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("io,wt", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("groups,per,cols", [(2, 1, 64), (7, 5, 200), (3, 100, 1111), (64, 3, 1024), (700, 2, 72), (5, 33, 2048),
                                             (4, 9, 4097), (2, 20, 8192), (3, 3, 9000), (300, 11, 333), (2, 1500, 256), (2, 700, 1001)])
def test_layernorm_by_groups(groups, per, cols, io, wt):
    rows = groups * per
    x, gy, gh = ((randn(groups + cols + k, rows, cols) + 1).to(io) for k in range(3))
    w, b = affine(rows, cols, groups, wt, cols + groups)
    for add_one, p, r in ((True, 0.0, None), (False, 0.1, gh)):
        h, mean, rstd = check_norm(x, r, w, b, add_one, p)
        check_norm_backward(gy, h, mean, rstd, w, gh, add_one, p)


@pytest.mark.gpu
@pytest.mark.parametrize("io", TYPES)
@pytest.mark.parametrize("rows,cols", [(9000, 512), (5000, 2048), (3000, 4096), (700, 8192), (3001, 1001), (900, 4099)])
def test_layernorm_of_many_rows(rows, cols, io):
    x, r, gy, gh = (randn(rows + cols + k, rows, cols).to(io) for k in range(4))
    w, b = affine(rows, cols, 1, io, cols)
    h, mean, rstd = check_norm(x, r, w, b, False, 0.0)
    check_norm_backward(gy, h, mean, rstd, w, gh, False, 0.0)


@pytest.mark.gpu
def test_layernorm_edges():
    """A mean far above the deviations, constant rows, rows that are no numbers, no rows, strides of zero."""
    x = randn(1, 40, 1024) * 0.01 + 1000
    check_norm(x, None, None, None, False, 0.0)
    x[3] = 5.0
    x[4] = 0.0
    y, _, _, rstd = B.prm_layernorm(x, eps=EPS)
    assert torch.all(y[3:5] == 0) and abs(float(rstd[4]) - 1000) < 1e-3
    y0 = y.clone()
    x[7, 5], x[8, 0] = float("nan"), float("inf")
    y, _, _, _ = B.prm_layernorm(x, eps=EPS)
    assert torch.all(torch.isnan(y[7])) and not torch.any(torch.isfinite(y[8]))
    rest = [i for i in range(40) if i not in (7, 8)]
    assert torch.equal(y[rest], y0[rest])
    y, h, mean, rstd = B.prm_layernorm(x[:0], torch.ones(1024, device="cuda"), residual=x[:0])
    assert y.shape == h.shape == (0, 1024) and mean.shape == (0,)
    _, _, gw, gb = B.prm_layernorm_backward(x[:0], x[:0], mean, rstd, torch.ones(3, 1024, device="cuda"))
    assert gw.shape == (3, 1024) and torch.all(gw == 0) and torch.all(gb == 0)
    same = randn(5, 1, 1024).expand(6, 1024)
    check_norm(same, same, torch.ones(1, 1024, device="cuda").expand(2, 1024), None, False, 0.0)


@pytest.mark.gpu
def test_layernorm_beyond_32_bits_of_offsets():
    """The last rows of a stream of more than 2^31 elements, on both sides of the pass."""
    rows, cols = 140000, 16384
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-40:] = randn(1, 40, cols).to(torch.bfloat16)
    x[:-40] = 1
    w = torch.ones(cols, device="cuda")
    y, _, mean, rstd = B.prm_layernorm(x, w)
    ry, rm, rr, size = R.norm(x[-40:], w, None, EPS)
    close(y[-40:], ry, 200 * R.F32 * size + 1.01 * R.BF16 * ry.abs(), "y")
    close(mean[-40:], rm, 100 * R.F32 * x[-40:].double().abs().mean(1), "mean")
    del y
    gx, _, gw, gb = B.prm_layernorm_backward(x, x, mean, rstd, w)
    rx, _, _, sx, _, _ = R.norm_backward(x[-40:], x[-40:], mean[-40:], rstd[-40:], w)
    close(gx[-40:], rx, 100 * R.F32 * sx + 1.01 * R.BF16 * rx.abs(), "grad_x")


@pytest.mark.gpu
def test_layernorm_refusals():
    x = randn(1, 6, 64)
    w = torch.ones(64, device="cuda")
    for bad in (dict(weight=w[:32]), dict(weight=torch.ones(4, 64, device="cuda")), dict(weight=w, bias=w.bfloat16()),
                dict(weight=w.half()), dict(residual=x[:3]), dict(p=1.0), dict(p=0.5, counter=torch.zeros(1, device="cuda")),
                dict(weight=w.cpu()), dict(bias=torch.ones(2, 64, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            B.prm_layernorm(x, **bad)
    with pytest.raises(B.PrmError):
        B.prm_layernorm(x, w, eps=-1.0)


# ------------------------------------------------------- loss of a linear head

def head_inputs(n, d, vocab, how, seed, scale=1.5):
    x = laid(randn(seed, n, d).to(torch.bfloat16), "padded" if how == "padded" else "dense")
    W = (randn(seed + 1, d, vocab) * scale * d ** -0.5).to(torch.bfloat16)
    if how == "out_in":
        W = W.t().contiguous().t()
    elif how == "padded":
        W = laid(W, "ragged")
    labels = torch.randint(0, vocab, (n,), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    if n > 2:
        labels[1], labels[n // 2], labels[n - 1] = -100, vocab, vocab - 1
    return x, W, labels


def check_head(x, W, labels, gl):
    n = len(x)
    loss, lse = B.prm_head_loss(x, W, labels)
    rl, rs, off, gx, gw, bx, bw = R.head(x, W, labels, gl)
    # a logit's error, the approximate exponentials' (2^-22 each), the logarithm's and the last roundings'
    room = 2 * off + 2.0 ** -20 + 4 * R.F32 * rs.abs()
    close(lse, rs, room, "lse")
    close(loss, rl, 2 * room, "loss")
    live = (labels >= 0) & (labels < W.shape[1])
    assert torch.all(loss[~live] == 0)
    got_x, got_w = B.prm_head_loss_backward(gl, x, W, labels, lse)
    assert got_w.shape == W.shape
    tiny = 1e-30
    close(got_x, gx, 1.02 * bx + 1.01 * R.BF16 * gx.abs() + tiny, "grad_x")
    close(got_w, gw, 1.02 * bw + 1.01 * R.BF16 * gw.abs() + tiny, "grad_w")
    # each entry of G and each result is rounded by itself, at most 2^-8 / sqrt(3) in the root of the mean square if a
    # value is anywhere in its binade: few rows and columns do not average
    if n >= 64 and x.shape[1] >= 64 and W.shape[1] >= 64:
        for got, ref in ((got_x, gx), (got_w, gw)):
            assert float((got.double() - ref).norm() / ref.norm()) < R.BF16 * (2 / 3) ** 0.5
    assert torch.all(got_x[~live] == 0)
    only_x, none = B.prm_head_loss_backward(gl, x, W, labels, lse, need_weight=False)
    assert none is None and torch.equal(only_x, got_x)
    none, only_w = B.prm_head_loss_backward(gl, x, W, labels, lse, need_x=False)
    assert none is None and torch.equal(only_w, got_w)


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["in_out", "out_in", "padded"])
@pytest.mark.parametrize("n,d,vocab", [(1, 8, 1), (1, 1, 5), (1, 64, 300), (3, 100, 77), (2, 512, 2500), (130, 72, 129), (257, 320, 1000),
                                       (64, 1000, 5003), (600, 1024, 4096), (1000, 513, 771), (31, 4096, 10000)])
def test_head_loss_and_gradient(n, d, vocab, how):
    x, W, labels = head_inputs(n, d, vocab, how, n + d)
    check_head(x, W, labels, torch.exp(randn(n, n)) * 1e-3)


@pytest.mark.gpu
def test_head_loss_of_a_mean():
    """The rows' factor is common: it stays out of G, and a mean over any number of rows has no error from it."""
    x, W, labels = head_inputs(777, 256, 2000, "in_out", 5)
    check_head(x, W, labels, torch.full((777,), 1 / 773, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["in_out", "out_in"])
def test_head_gradient_in_pieces(how):
    """So many rows that G is made for one half of the vocabulary after the other; the second is narrower."""
    x, W, labels = head_inputs(131072, 64, 4000, how, 6)
    check_head(x, W, labels, torch.full((131072,), 2.0 ** -17, device="cuda"))


@pytest.mark.gpu
def test_head_gradient_in_pieces_of_a_wide_vocabulary():
    """Few enough rows that their common factor is found by the first piece's product; the second reads it."""
    n, d, vocab = 2000, 40, 140001
    x, W, labels = head_inputs(n, d, vocab, "out_in", 11)
    gl = torch.exp(randn(12, n)) / n
    loss, lse = B.prm_head_loss(x, W, labels)
    gx, gw = B.prm_head_loss_backward(gl, x, W, labels, lse)
    rl, rs, off, rx, rw, bx, bw = R.head(x, W, labels, gl, part=500)
    room = 2 * off + 2.0 ** -20 + 4 * R.F32 * rs.abs()
    close(loss, rl, 2 * room, "loss")
    close(gx, rx, 1.02 * bx + 1.01 * R.BF16 * rx.abs() + 1e-30, "grad_x")
    close(gw, rw, 1.02 * bw + 1.01 * R.BF16 * rw.abs() + 1e-30, "grad_w")


@pytest.mark.gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_head_weight_beyond_32_bits_of_offsets(transposed):
    """A weight of more than 2^31 elements: the loss, and the last of its gradient."""
    n, d, vocab = 70, 16400, 131080
    x = randn(1, n, d).to(torch.bfloat16)
    shape = (vocab, d) if transposed else (d, vocab)
    W = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, d ** -0.5, generator=torch.Generator(device="cuda").manual_seed(2))
    W = W.t() if transposed else W
    labels = torch.arange(n, device="cuda") * 1000 + vocab - 1000 * n
    logits = torch.zeros(n, vocab, dtype=torch.float64, device="cuda")
    size = 0.0
    for k in range(0, d, 1024):
        logits += x[:, k:k + 1024].double() @ W[k:k + 1024].double()
        size += float((x[:, k:k + 1024].double().abs() @ W[k:k + 1024, ::97].double().abs()).amax())
    lse = torch.logsumexp(logits, 1)
    off = 1.1 * (d / 16 + 4) * 2.0 ** -23 * size          # every 97th column's largest sum of magnitudes, and a tenth
    loss, got = B.prm_head_loss(x, W, labels)
    room = 2 * off + 2.0 ** -20 + 4 * R.F32 * lse.abs()
    close(got, lse, room, "lse")
    close(loss, lse - logits.gather(1, labels[:, None])[:, 0], 2 * room, "loss")
    gl = torch.full((n,), 1 / 64, device="cuda")
    _, gw = B.prm_head_loss_backward(gl, x, W, labels, got, need_x=False)
    g = torch.exp(logits - lse[:, None])
    g[torch.arange(n, device="cuda"), labels] -= 1
    g /= 64
    want = x[:, -9:].double().t() @ g
    dg = R.BF16 * g.abs() + (2 * off + 2.0 ** -19) / 64 * torch.exp(logits - lse[:, None])
    close(gw[-9:], want, 1.02 * x[:, -9:].double().abs().t() @ dg + 1.01 * R.BF16 * want.abs() + 1e-30, "grad_w")


@pytest.mark.gpu
def test_head_loss_in_parts_of_rows():
    """So many columns that the rows' partial sums are joined before all rows have been seen."""
    n, d, vocab = 9001, 16, 262144
    x, W, labels = head_inputs(n, d, vocab, "in_out", 7)
    loss, lse = B.prm_head_loss(x, W, labels)
    rl, rs, off, *_ = R.head(x, W, labels, part=1024)
    room = 2 * off + 2.0 ** -20 + 4 * R.F32 * rs.abs()
    close(lse, rs, room, "lse")
    close(loss, rl, 2 * room, "loss")


@pytest.mark.gpu
def test_head_loss_of_far_logits():
    """Logits of some hundreds, either sign, equal ones, and a vocabulary's column of -infinities."""
    for scale in (200.0, 1e-6):
        x, W, labels = head_inputs(70, 128, 900, "in_out", 8, scale)
        check_head(x, W, labels, torch.ones(70, device="cuda"))
    x = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    W = torch.full((64, 600), -40.0, dtype=torch.bfloat16, device="cuda")
    labels = torch.tensor([0, 599, 300, -1], device="cuda")
    loss, lse = B.prm_head_loss(x, W, labels)
    want = -2560 + torch.log(torch.tensor(600.0, dtype=torch.float64))
    assert torch.all((lse.double() - want.cuda()).abs() < 2560 * 2 * R.F32 + 2.0 ** -20)
    W[:, :256] = float("-inf")
    loss, lse = B.prm_head_loss(x, W, labels)
    want = -2560 + torch.log(torch.tensor(344.0, dtype=torch.float64))
    assert torch.all((lse.double() - want.cuda()).abs() < 2560 * 2 * R.F32 + 2.0 ** -20)
    assert float(loss[0]) == float("inf") and float(loss[3]) == 0


@pytest.mark.gpu
def test_head_loss_of_what_is_no_number():
    x, W, labels = head_inputs(300, 64, 700, "in_out", 9)
    loss, lse = B.prm_head_loss(x, W, labels)
    gl = torch.ones(300, device="cuda")
    gx, _ = B.prm_head_loss_backward(gl, x, W, labels, lse)
    x[10, 3], x[290, 0] = float("nan"), float("inf")
    loss2, lse2 = B.prm_head_loss(x, W, labels)
    bad = torch.zeros(300, dtype=torch.bool, device="cuda")
    bad[[10, 290]] = True
    assert not torch.any(torch.isfinite(loss2[bad])) and torch.equal(loss2[~bad], loss[~bad]) and torch.equal(lse2[~bad], lse[~bad])
    gx2, _ = B.prm_head_loss_backward(gl, x, W, labels, lse2)
    assert torch.equal(gx2[~bad], gx[~bad]) and not torch.any(torch.isfinite(gx2[bad]))


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,vocab,how", [(5, 64, 300, "in_out"), (300, 100, 700, "out_in"), (2500, 77, 513, "padded"), (131072, 8, 4000, "in_out")])
def test_head_gradient_ignores_what_rows_without_a_part_hold(n, d, vocab, how):
    """Padding that is no number: rows without a label, and rows whose loss has the gradient 0."""
    x, W, labels = head_inputs(n, d, vocab, how, n)
    gl = torch.exp(randn(n, n))
    labels[::3] = -100
    gl[1::7] = 0
    dead = (labels < 0) | (labels >= vocab) | (gl == 0)
    x[dead] = 0
    _, lse = B.prm_head_loss(x, W, labels)
    want = B.prm_head_loss_backward(gl, x, W, labels, lse)
    for junk in (float("nan"), float("inf"), -3e38):
        x[dead] = junk
        loss, lse = B.prm_head_loss(x, W, labels)
        assert torch.all(torch.isfinite(loss[~dead])) and torch.all(loss[(labels < 0) | (labels >= vocab)] == 0)
        got = B.prm_head_loss_backward(gl, x, W, labels, lse)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.all(got[0][dead] == 0)


@pytest.mark.gpu
def test_head_loss_without_rows_or_labels():
    x, W, labels = head_inputs(20, 64, 700, "in_out", 10)
    loss, lse = B.prm_head_loss(x[:0], W, labels[:0])
    assert loss.shape == lse.shape == (0,)
    gx, gw = B.prm_head_loss_backward(loss, x[:0], W, labels[:0], lse)
    assert gx.shape == (0, 64) and torch.all(gw == 0)
    none = torch.full_like(labels, -100)
    loss, lse = B.prm_head_loss(x, W, none)
    gx, gw = B.prm_head_loss_backward(torch.full((20,), float("nan"), device="cuda"), x, W, none, lse)
    assert torch.all(loss == 0) and torch.all(gx == 0) and torch.all(gw == 0)


@pytest.mark.gpu
def test_head_refusals():
    x, W, labels = head_inputs(20, 64, 700, "in_out", 10)
    for args in ((x, W, labels.int()), (x, W, labels[:5]), (x, W[:32], labels), (x.float(), W.float(), labels), (x, W[:, :0], labels),
                 (x, W, labels.cpu()), (x.cpu(), W, labels), (x[0], W, labels)):
        with pytest.raises((ValueError, TypeError)):
            B.prm_head_loss(*args)


@pytest.mark.gpu
def test_no_wait_ran_out():
    assert B.prm_q8_status() == B.PRM_OK
