"""What the gradients of layer norm and the head's loss accept, and the scratch that they ask for, decided before anything touches the
device."""

import pytest

from paper_2608_20818_b200 import binding as B

P = 1 << 20                     # an address that is never read


def layernorm_backward(rows, cols, per, nbytes, **change):
    a = dict(gy=P, ldgy=cols, h=P, ldh=cols, mean=P, rstd=P, w=P, ldw=cols, gh=None, ldgh=0, rows=rows, cols=cols, per=per, io=0, wfp32=0,
             one=0, p=0.0, seed=1, offset=0, counter=None, gr=P, ldgr=cols, gx=None, ldgx=0, gw=P, gb=P, scratch=P, nbytes=nbytes,
             stream=None)
    return B.lib().prm_layernorm_backward(*{**a, **change}.values())


@pytest.mark.parametrize("rows,cols,per,code", [
    (4000000, 64, 1, B.PRM_ERR_WORKSPACE), (1 << 28, 256, 1, B.PRM_ERR_WORKSPACE), ((1 << 30) - 1, 8, 1, B.PRM_ERR_WORKSPACE),
    (1 << 28, 100, 8, B.PRM_ERR_WORKSPACE), (1 << 30, 100000, 1, B.PRM_ERR_SHAPE), (2 ** 31 - 8, 64, 4, B.PRM_ERR_WORKSPACE), (2 ** 31 - 1, 8, 1, B.PRM_ERR_SHAPE),
])
def test_layernorm_gradient_takes_as_many_groups_as_a_launch_has_blocks(rows, cols, per, code):
    """No scratch is given, so that what is accepted ends there."""
    assert layernorm_backward(rows, cols, per, 0) == code
