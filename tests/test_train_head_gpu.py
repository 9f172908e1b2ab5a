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
