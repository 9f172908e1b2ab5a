"""Refusals of the 8-bit operators that are decided before anything touches the device."""

import pytest

from paper_2608_20818_b200 import binding as B

P = 1 << 20                     # an address that is never read


def quantize(**change):
    args = dict(x=P, ldx=64, rows=4, cols=64, io=0, fmt=0, fr=None, fc=None, qr=None, ldqr=0, sr=None, qc=P, ldqc=64, sc=P,
                scratch=P, nbytes=1 << 20, stream=None)
    return B.lib().prm_quantize_q8(*{**args, **change}.values())


@pytest.mark.parametrize("off", [1, 2, 4, 8, 12])
def test_quantizer_scratch_is_read_in_pieces_of_16_bytes(off):
    assert quantize(scratch=P + off) == B.PRM_ERR_ALIGN
    # not read without codes by column: the next check answers
    assert quantize(scratch=P + off, qr=P, sr=P, ldqr=64, qc=None, x=None) == B.PRM_ERR_ARG
