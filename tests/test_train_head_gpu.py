"""The loss of a linear head and its gradient where sizes or values are extreme, against 64 bits."""

import pytest
import torch

import train_reference as R
from paper_2608_20818_b200 import binding as B


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def close(got, want, room, what):
    bad = (got.double() - want).abs() - room
    assert torch.all(bad <= 0), (what, float(bad.max()))


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [3069441, 3069550])
def test_gradient_whose_last_piece_has_fewer_stages_than_parts(vocab):
    """110 pieces of the vocabulary, two parts of k in each but the last, which has 1 or 110 columns."""
    n, d = 9472, 24
    x = randn(1, n, d).to(torch.bfloat16)
    W = (randn(2, d, vocab) * d ** -0.5).to(torch.bfloat16)
    labels = torch.randint(0, vocab, (n,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    labels[::5] = torch.arange(len(labels[::5]), device="cuda") % 110 + vocab - 110          # in the last piece, or beside it
    labels[7::50] = -1
    gl = torch.exp(randn(4, n)) / n
    _, lse = B.prm_head_loss(x, W, labels)
    gx, gw = B.prm_head_loss_backward(gl, x, W, labels, lse)
    assert B.prm_q8_status() == B.PRM_OK
    _, _, _, rx, rw, bx, bw = R.head(x, W, labels, gl, part=128)
    close(gx, rx, 1.02 * bx + 1.01 * R.BF16 * rx.abs() + 1e-30, "grad_x")
    close(gw, rw, 1.02 * bw + 1.01 * R.BF16 * rw.abs() + 1e-30, "grad_w")


def confident(n, d, vocab, size, seed):
    """Rows along their labels' columns: their logits are about `size`, the others' some size / sqrt(d)."""
    W = randn(seed, d, vocab).to(torch.bfloat16)
    labels = torch.randint(0, vocab, (n,), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    return (W.t()[labels].float() * (size / d)).to(torch.bfloat16), W, labels


@pytest.mark.gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n", [1, 40, 512])
@pytest.mark.parametrize("d", [64, 1024, 4096])
@pytest.mark.parametrize("size", [10.0, 20.0, 50.0, 100.0])
def test_loss_of_confident_rows(n, d, size, transposed):
    """No loss is below 0, and where nothing but the label counts it is 0: what else there is, less than 2^-25 in all, leaves a
    sum of 1 as it is."""
    x, W, labels = confident(n, d, 2000, size, n + d)
    W = W.t().contiguous().t() if transposed else W
    loss, lse = B.prm_head_loss(x, W, labels)
    want, want_lse, off, *_ = R.head(x, W, labels)
    assert torch.all(loss >= 0)
    sure = want < 2.0 ** -26
    assert torch.all(loss[sure] == 0) and (size < 50 or d < 1024 or bool(torch.all(sure)))
    # the other logits' shares are as far off as two logits and the exponential's rounding; a number is added to the sum 128 times
    # at most (a thread's 32 and 3, the rows' parts), then the logarithm
    close(loss, want, torch.expm1(want) * (2 * off + 2.0 ** -20) + 128 * R.F32 * (1 + want), "loss")
    close(lse, want_lse, off + 2.0 ** -20 + 2 * R.F32 * want_lse.abs(), "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n,d,size", [(512, 4096, 10.0), (512, 4096, 14.0), (130, 8200, 14.0), (200, 1000, 14.0)])
def test_gradient_of_confident_rows(n, d, size, transposed):
    """The gradient's logits are those that lse was made of, so that what is off in them changes 1 - p by its own share only:
    the label's entry of G has no error of the size of a logit's, however long its sum."""
    x, W, labels = confident(n, d, 2000, size, d)
    W = W.t().contiguous().t() if transposed else W
    _, lse = B.prm_head_loss(x, W, labels)
    gl = torch.exp(randn(5, n)) / n
    gx, gw = B.prm_head_loss_backward(gl, x, W, labels, lse)
    xd, Wd, g1 = x.double(), W.double(), gl.double()[:, None]
    logits = xd @ Wd
    p = torch.softmax(logits, 1)
    rows = torch.arange(n, device="cuda")
    rest = p.sum(1) - p[rows, labels]                      # 1 - p of the label
    g = p.clone()
    g[rows, labels] = -rest
    off = (d / 16 + 4) * 2.0 ** -23 * (xd.abs() @ Wd.abs()).amax(1, keepdim=True)
    # an entry's rounding to bf16, the logits', and the exponential's and lse's own roundings, which p carries whole
    dg = R.BF16 * g.abs() + g.abs() * 2 * off + p * (2.0 ** -21 + 2 * R.F32 * lse.double().abs()[:, None])
    g, dg = g * g1, dg * g1
    rx, rw = g @ Wd.t(), xd.t() @ g
    close(gx, rx, 1.02 * dg @ Wd.t().abs() + 1.01 * R.BF16 * rx.abs() + 1e-30, "grad_x")
    close(gw, rw, 1.02 * xd.t().abs() @ dg + 1.01 * R.BF16 * rw.abs() + 1e-30, "grad_w")


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,vocab", [(20, 64, 700), (300, 100, 1003), (2100, 77, 513)])
def test_gradient_of_x_alone_keeps_to_its_scratch(n, d, vocab):
    """The least scratch, with what lies behind it untouched; the same bits as with the weight's gradient."""
    L = B.lib()
    x, W = randn(1, n, d).to(torch.bfloat16), randn(2, vocab, d).to(torch.bfloat16)
    labels, gl = torch.arange(n, device="cuda") % vocab, torch.exp(randn(3, n))
    _, lse = B.prm_head_loss(x, W.t(), labels)
    want, _ = B.prm_head_loss_backward(gl, x, W.t(), labels, lse)
    nbytes = L.prm_head_loss_backward_scratch_bytes(n, d, vocab) - L.prm_head_loss_copy_bytes(n, d)
    if d % 8:
        nbytes += L.prm_head_loss_copy_bytes(n, d) + L.prm_head_loss_copy_bytes(vocab, d)
    scratch = torch.full((nbytes + 4096,), 77, dtype=torch.uint8, device="cuda")
    gx = torch.empty_like(x)
    code = L.prm_head_loss_backward(gl.data_ptr(), x.data_ptr(), d, W.data_ptr(), d, 1, labels.data_ptr(), lse.data_ptr(), n, d, vocab,
                                    gx.data_ptr(), d, None, d, scratch.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
    assert code == B.PRM_OK and torch.equal(gx, want) and torch.all(scratch[nbytes:] == 77)
    assert torch.equal(B.prm_head_loss_backward(gl, x, W.t(), labels, lse, need_weight=False)[0], want)


def rounded(got, want, longest, chunks, what):
    """Sums of one sign: in fp32 each is off by what is cut off at each step of 16 of the longest sum that is kept in one place,
    and by a rounding for each of those sums, relative to itself.  Rounding to bf16 keeps the order of numbers, so that the result
    lies between the roundings of the ends of that range.  (How results' roundings average says nothing: want lies on
    a grid like bf16's own here, less n / vocab, so that all of them may go the same way.)"""
    off = (longest / 16 + 4) * 2.0 ** -23 + (chunks + 4) * R.F32
    low, high = (want * (1 - off)).to(torch.bfloat16), (want * (1 + off)).to(torch.bfloat16)
    assert torch.all((got >= low) & (got <= high)), (what, float(((got.double() - want) / want).abs().max()))


@pytest.mark.gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n", [9000, 1 << 17, 1 << 20])
def test_weight_s_gradient_of_many_rows(n, transposed):
    """All logits 0, so that G is 1/256 and 1/256 - 1, exactly: grad_W's sums are over as many terms as there are rows."""
    d, vocab = 64, 256
    x = ((1 + 0.1 * randn(1, n, d)) * (1 + torch.arange(d, device="cuda") / d)).to(torch.bfloat16)
    W = torch.zeros(vocab, d, dtype=torch.bfloat16, device="cuda").t() if transposed else torch.zeros(d, vocab, dtype=torch.bfloat16, device="cuda")
    labels = torch.randint(0, 4, (n,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    _, lse = B.prm_head_loss(x, W, labels)
    _, gw = B.prm_head_loss_backward(torch.ones(n, device="cuda"), x, W, labels, lse, need_x=False)
    want = x.double().sum(0) / 256
    longest = n if n <= 32768 else 8192
    rounded(gw[:, 4:], want[:, None].expand(d, vocab - 4), longest, n // longest, "columns without a label")
    hot = torch.stack([x[labels == v].double().sum(0) for v in range(4)], 1)
    close(gw[:, :4], want[:, None] - hot, ((longest / 16 + 4) * 2.0 ** -23 + (n // longest + 4) * R.F32) * (want[:, None] + hot) +
          1.01 * R.BF16 * (want[:, None] - hot).abs(), "columns with labels")


@pytest.mark.gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n,vocab", [(64, 1 << 15), (64, 1 << 21), (600, 1 << 18)])
def test_rows_gradient_of_a_long_vocabulary(n, vocab, transposed):
    """Rows of zeros, so that G is 1 / vocab, exactly, but for the label: its column is 0."""
    d = 64
    W = ((1 + 0.1 * randn(1, vocab, d)) * (1 + torch.arange(d, device="cuda") / d)).to(torch.bfloat16)
    W[:n] = 0
    want = (W.double().sum(0) / vocab)[None].expand(n, d)
    W = W.t() if transposed else W.t().contiguous()
    x = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    labels = torch.arange(n, device="cuda")
    _, lse = B.prm_head_loss(x, W, labels)
    gx, _ = B.prm_head_loss_backward(torch.ones(n, device="cuda"), x, W, labels, lse, need_weight=False)
    longest = vocab if vocab <= 32768 else 8192
    rounded(gx, want, longest, vocab // longest, "grad_x")
