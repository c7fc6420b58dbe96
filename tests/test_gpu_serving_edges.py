"""The serving operators where calls that the header allows are out of the ordinary: a prefix alone, tokens that a table has no room for."""

import pytest
import torch

from layers_harness import DEV
from paper_1711_07240_amd import block as B
from serving_harness import Attention
from test_gpu_block import _off

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


# (few rows and keys, keys dealt to workgroups, few rows of float, tiles of one request's rows, those that workgroups share)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fresh,held,more,prefix,heads,D", [([4, 1, 2], [16, 7, 16], [2, 0, 1], 30, (4, 2), 64), ([100, 1], [64, 3], [36, 0], 0, (4, 2), 32),
                                                            ([2, 1, 3, 0], [1280, 30, 1280, 5], [1, 0, 70, 0], 0, (8, 2), 64), ([1, 1], [1280, 9], [5, 0], 700, (2, 2), 128),
                                                            ([5, 40], [2048, 2048], [4, 39], 900, (6, 2), 40), ([300, 1, 511, 700], [320, 9, 704, 704], [200, 0, 1, 699], 200, (16, 8), 32),
                                                            ([700, 700, 3, 500], [1408, 1408, 7, 1408], [5, 1408, 0, 130], 300, (16, 8), 64)])
def test_tokens_that_the_table_has_no_room_for(fresh, held, more, prefix, heads, D, dtype):
    """They count where a row's own token is, and are not seen."""
    a = Attention(dtype, fresh, held, prefix, 16, *heads, D, extra=0, pad=1)
    assert a.most * 16 == max(held)
    a.lengths = [n + m for n, m in zip(held, more)]
    a.check(*a.call(), rows=[0, 1, 2, 3, 4, 15, 35, 36, 39, 63, 64, 99, 127, 128, 299, 499, 510, 511, 699])
    if set(fresh) == {1}:
        a = Attention(dtype, fresh, held, prefix, 16, *heads, D, extra=0)
        a.lengths = [n + m for n, m in zip(held, more)]
        a.check(*a.call(single=True))


@pytest.mark.parametrize("dtype,tol", [("f32", 2e-5), ("bf16", 3e-2)])
def test_a_request_outgrows_its_table(dtype, tol):
    """The tokens that still find a place are answered as ever, in that step too."""
    blk = B.Block(channels=64, heads=2, head_size=32, width=96, positions=128, dtype=dtype)
    x = torch.randn(10, 64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).to(blk.dt)
    want = blk.forward(x, 1).cpu()
    pages = B.Pages(blk, requests=1, rows=5, pages=20, page=2, most=4)
    pages.fresh.fill_(5)
    assert _off(pages.step(x[:5]), want[:5]) <= tol and pages.taken.tolist() == [3, 0]
    second = pages.step(x[5:])
    assert pages.slots.tolist()[3:] == [-1, -1] and pages.taken.tolist() == [4, 2]
    assert _off(second[:3], want[5:8]) <= tol
