"""The serving operators where calls that the header allows are out of the ordinary: a prefix alone."""

import pytest
import torch

from serving_harness import Attention

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16"]


# (heads of 32 and 64 key heads make more tiles of the prefix's rows than half of the compute units: one part of it, which is the result)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fresh,Hq,Hk,D,prefix", [([300], 64, 64, 32, 600), ([1] * 300, 64, 64, 32, 600), ([90, 0, 200, 1], 128, 64, 40, 1100), ([1] * 3, 8, 2, 64, 9000),
                                                  ([40, 2], 8, 8, 80, 513), ([1], 4, 4, 128, 2000)])
def test_a_prefix_alone(fresh, Hq, Hk, D, prefix, dtype):
    """max_pages = 0: tables of no requests' own."""
    a = Attention(dtype, fresh, [0] * len(fresh), prefix, 16, Hq, Hk, D, extra=0, pad=2)
    assert a.most == 0
    rows = [0, 1, 63, 64, 127, 128, 199, 299]
    a.check(*a.call(), rows=rows)
    if max(fresh) == 1:
        a = Attention(dtype, fresh, [0] * len(fresh), prefix, 16, Hq, Hk, D, extra=0)
        first = a.call(single=True)
        a.check(*first, rows=rows)
        assert all(torch.equal(x, y) for x, y in zip(first, a.call(single=True)))
