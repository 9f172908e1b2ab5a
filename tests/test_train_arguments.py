"""Dropout, layer norm and the head's loss: the generator's published answers, refusals that are decided before anything touches
the device, and the arithmetic of the scratch's sizes."""

import numpy as np
import pytest
import torch

import train_reference as R
from paper_2608_20818_b200 import binding as B

P = 1 << 20                     # an address that is never read


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_oracle_generator_gives_the_published_words(counter, key, words):
    assert tuple(int(v) for v in R.philox(counter, key)) == words


def test_oracle_keeps_the_share_that_it_should():
    k = R.keep(400, 1001, 0.3, 12345678901234567890, 2 ** 40 + 7).double().mean()
    assert abs(float(k) - 0.7) < 5 * (0.21 / 400400) ** 0.5          # five standard deviations


def dropout(**change):
    a = dict(x=P, ldx=64, r=None, ldr=0, rows=4, cols=64, io=0, p=0.1, seed=1, offset=0, counter=None, out=P, ldo=64, stream=None)
    return B.lib().prm_dropout(*{**a, **change}.values())


@pytest.mark.parametrize("change,code", [
    (dict(p=1.0), B.PRM_ERR_ARG), (dict(p=-0.1), B.PRM_ERR_ARG), (dict(p=float("nan")), B.PRM_ERR_ARG),
    (dict(rows=-1), B.PRM_ERR_ARG), (dict(x=None), B.PRM_ERR_ARG), (dict(out=None), B.PRM_ERR_ARG),
    (dict(cols=-1), B.PRM_ERR_SHAPE), (dict(cols=2 ** 31), B.PRM_ERR_SHAPE), (dict(rows=2 ** 31), B.PRM_ERR_SHAPE),
    (dict(ldo=63), B.PRM_ERR_SHAPE), (dict(ldx=-1), B.PRM_ERR_SHAPE), (dict(r=P, ldr=-1), B.PRM_ERR_SHAPE),
    (dict(x=P + 1), B.PRM_ERR_ALIGN), (dict(io=1, out=P + 2), B.PRM_ERR_ALIGN), (dict(counter=P + 4), B.PRM_ERR_ALIGN),
    (dict(rows=0, x=None, out=None), B.PRM_OK), (dict(cols=0, ldo=0, x=None), B.PRM_OK),
])
def test_dropout_refusals(change, code):
    assert dropout(**change) == code


def layernorm(**change):
    a = dict(x=P, ldx=64, r=None, ldr=0, w=P, ldw=64, b=P, ldb=64, rows=4, cols=64, per=4, io=0, wfp32=0, one=0, eps=1e-6, p=0.0,
             seed=1, offset=0, counter=None, h=None, ldh=0, y=P, ldy=64, mean=P, rstd=P, stream=None)
    return B.lib().prm_layernorm(*{**a, **change}.values())


@pytest.mark.parametrize("change,code", [
    (dict(eps=-1.0), B.PRM_ERR_ARG), (dict(eps=float("nan")), B.PRM_ERR_ARG), (dict(p=1.0), B.PRM_ERR_ARG),
    (dict(rows=-1), B.PRM_ERR_ARG), (dict(per=0), B.PRM_ERR_ARG), (dict(x=None), B.PRM_ERR_ARG), (dict(y=None), B.PRM_ERR_ARG),
    (dict(mean=None), B.PRM_ERR_ARG), (dict(rstd=None), B.PRM_ERR_ARG), (dict(r=P, ldr=64, ldh=64), B.PRM_ERR_ARG),
    (dict(p=0.5, ldh=64), B.PRM_ERR_ARG), (dict(cols=0), B.PRM_ERR_SHAPE), (dict(rows=2 ** 31), B.PRM_ERR_SHAPE),
    (dict(ldy=63), B.PRM_ERR_SHAPE), (dict(ldw=-1), B.PRM_ERR_SHAPE), (dict(p=0.5, h=P, ldh=63), B.PRM_ERR_SHAPE),
    (dict(y=P + 1), B.PRM_ERR_ALIGN), (dict(wfp32=1, b=P + 2), B.PRM_ERR_ALIGN), (dict(mean=P + 2), B.PRM_ERR_ALIGN),
    (dict(counter=P + 4), B.PRM_ERR_ALIGN), (dict(rows=0, x=None, y=None), B.PRM_OK),
])
def test_layernorm_refusals(change, code):
    assert layernorm(**change) == code


def layernorm_backward(**change):
    a = dict(gy=P, ldgy=64, h=P, ldh=64, mean=P, rstd=P, w=P, ldw=64, gh=None, ldgh=0, rows=4, cols=64, per=4, io=0, wfp32=0,
             one=0, p=0.0, seed=1, offset=0, counter=None, gr=P, ldgr=64, gx=None, ldgx=0, gw=P, gb=P, scratch=P, nbytes=1 << 30,
             stream=None)
    return B.lib().prm_layernorm_backward(*{**a, **change}.values())


@pytest.mark.parametrize("change,code", [
    (dict(p=1.5), B.PRM_ERR_ARG), (dict(per=0), B.PRM_ERR_ARG), (dict(gy=None), B.PRM_ERR_ARG), (dict(h=None), B.PRM_ERR_ARG),
    (dict(mean=None), B.PRM_ERR_ARG), (dict(rstd=None), B.PRM_ERR_ARG), (dict(gr=None), B.PRM_ERR_ARG),
    (dict(p=0.5, ldgx=64), B.PRM_ERR_ARG), (dict(scratch=None), B.PRM_ERR_ARG), (dict(cols=0), B.PRM_ERR_SHAPE),
    (dict(per=3), B.PRM_ERR_SHAPE), (dict(ldgr=63), B.PRM_ERR_SHAPE), (dict(p=0.5, gx=P, ldgx=63), B.PRM_ERR_SHAPE),
    (dict(nbytes=0), B.PRM_ERR_WORKSPACE), (dict(gw=P + 1), B.PRM_ERR_ALIGN), (dict(h=P + 1), B.PRM_ERR_ALIGN),
    (dict(scratch=P + 8), B.PRM_ERR_ALIGN), (dict(mean=P + 2), B.PRM_ERR_ALIGN), (dict(counter=P + 4), B.PRM_ERR_ALIGN),
])
def test_layernorm_backward_refusals(change, code):
    assert layernorm_backward(**change) == code


def head(**change):
    a = dict(x=P, ldx=64, w=P, ldw=128, t=0, labels=P, n=4, d=64, vocab=128, loss=P, lse=P, scratch=P, nbytes=1 << 30, stream=None)
    return B.lib().prm_head_loss(*{**a, **change}.values())


def head_backward(**change):
    a = dict(gl=P, x=P, ldx=64, w=P, ldw=128, t=0, labels=P, lse=P, n=4, d=64, vocab=128, gx=P, ldgx=64, gw=P, ldgw=128, scratch=P,
             nbytes=1 << 30, stream=None)
    return B.lib().prm_head_loss_backward(*{**a, **change}.values())


SHARED = [
    (dict(n=-1), B.PRM_ERR_SHAPE), (dict(d=0), B.PRM_ERR_SHAPE), (dict(vocab=0), B.PRM_ERR_SHAPE), (dict(vocab=2 ** 27 + 1, ldw=2 ** 28), B.PRM_ERR_SHAPE),
    (dict(n=2 ** 27 + 1), B.PRM_ERR_SHAPE), (dict(d=2 ** 27 + 1, ldx=2 ** 28), B.PRM_ERR_SHAPE),
    (dict(x=None), B.PRM_ERR_ARG), (dict(w=None), B.PRM_ERR_ARG), (dict(labels=None), B.PRM_ERR_ARG), (dict(lse=None), B.PRM_ERR_ARG),
    (dict(scratch=None), B.PRM_ERR_ARG), (dict(ldx=63), B.PRM_ERR_SHAPE), (dict(ldw=120), B.PRM_ERR_SHAPE), (dict(x=P + 1), B.PRM_ERR_ALIGN),
    (dict(w=P + 3), B.PRM_ERR_ALIGN), (dict(labels=P + 4), B.PRM_ERR_ALIGN),
    (dict(lse=P + 2), B.PRM_ERR_ALIGN), (dict(scratch=P + 8), B.PRM_ERR_ALIGN), (dict(nbytes=16), B.PRM_ERR_WORKSPACE),
]


@pytest.mark.parametrize("change,code", SHARED + [(dict(loss=None), B.PRM_ERR_ARG), (dict(n=0, x=None, loss=None), B.PRM_OK)])
def test_head_loss_refusals(change, code):
    assert head(**change) == code


@pytest.mark.parametrize("change,code", SHARED + [
    (dict(gl=None), B.PRM_ERR_ARG), (dict(ldgx=63), B.PRM_ERR_SHAPE), (dict(ldgw=127), B.PRM_ERR_SHAPE), (dict(gx=P + 1), B.PRM_ERR_ALIGN),
    (dict(gx=None, gw=None, x=None), B.PRM_OK), (dict(n=0, gw=None, x=None), B.PRM_OK),
])
def test_head_loss_backward_refusals(change, code):
    assert head_backward(**change) == code


@pytest.mark.parametrize("change", [dict(ldx=65), dict(x=P + 8), dict(w=P + 2), dict(ldw=132), dict(ldx=66, ldw=130)])
def test_head_copies_need_their_scratch(change):
    """An operand off 16 bytes is copied into scratch of its own: one byte less than that is refused."""
    L = B.lib()
    more = (L.prm_head_loss_copy_bytes(4, 64) if change.keys() & {"x", "ldx"} else 0) + \
        (L.prm_head_loss_copy_bytes(64, 128) if change.keys() & {"w", "ldw"} else 0)
    assert more >= 4 * 64 * 2
    assert head(nbytes=L.prm_head_loss_scratch_bytes(4, 64, 128) + more - 1, **change) == B.PRM_ERR_WORKSPACE
    assert head_backward(nbytes=L.prm_head_loss_backward_scratch_bytes(4, 64, 128) + more - 1, **change) == B.PRM_ERR_WORKSPACE


def test_head_scratch_is_bounded():
    """Neither direction asks for the logits: 128 MB forward unless 2048 rows need more, and backward G for a piece of 512 MB (or
    2048 columns), grad_x's sums (16 parts at most, with few rows), x once more and some padding."""
    L = B.lib()
    for n in (1, 7, 256, 8192, 65536, 1 << 20):
        for d in (8, 512, 4096):
            for vocab in (1, 1000, 32768, 262144, 1 << 21):
                parts = 2 * -(-vocab // 256)
                assert L.prm_head_loss_scratch_bytes(n, d, vocab) <= 256 + max(1 << 27, 2048 * parts * 8) + 4 * n
                g = L.prm_head_loss_backward_scratch_bytes(n, d, vocab)
                assert g <= 1024 + max(1 << 29, 2 * n * 2048) + 128 * n + 4 * n * (d + 3) * (16 if n <= 74 * 256 else 1) + 2 * n * d


def test_binding_refusals_without_a_device():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.prm_dropout(x, 0.1, 1)
    with pytest.raises(ValueError):
        B.prm_layernorm(x)
    with pytest.raises(ValueError):
        B.prm_head_loss(x, torch.zeros(8, 16, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(TypeError):
        B.prm_head_loss(x.float(), torch.zeros(8, 16), torch.zeros(4, dtype=torch.int64))
