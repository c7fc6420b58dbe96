"""Tensors of more planes than a launch has threads for are refused; done, a part of them would be left as it was, without an error.  Without a
GPU: refused calls never get to one."""

import pytest
import torch

from paper_1711_07240_amd import cgbn as L

# (a call that is wrongly taken would follow addresses that are none)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU")
P = 1 << 20


def _code(call, *args):
    try:
        call(*args)
    except L.CgbnError as e:
        return e.code
    return L.CGBN_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_planes_of_a_wavefront_each(dtype):
    """2^26 planes of 8 x 8 and more: 64 threads for each are 2^32."""
    for C, refused in ((1023, False), (1025, True)):
        size = (1 << 16, C, 8, 8, "NCHW")
        codes = (_code(L.cgbn_frozen_forward, P, *size, dtype, P, P, P, P, 1e-5, 2 * P, 0),
                 _code(L.cgbn_frozen_backward, P, *size, dtype, P, P, 1e-5, 2 * P, 0),
                 _code(L.cgbn_forward, P, *size, 1, P, P, 1e-5, 2 * P, 3 * P, 4 * P, dtype, 5 * P, 6 * P, 1 << 60, 0))
        assert all((code == 2) == refused and code != L.CGBN_OK for code in codes), codes
