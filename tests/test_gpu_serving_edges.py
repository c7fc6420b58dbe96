"""The serving operators where calls that the header allows are out of the ordinary: a prefix alone, tokens that a table has no room for, tokens
that get no place in the cache."""

import numpy as np
import pytest
import torch

from layers_harness import DEV, workspace
from paper_1711_07240_amd import block as B
from paper_1711_07240_amd import cgbn as L
from serving_harness import Attention, ints
from test_gpu_block import _off
from test_gpu_pages import _plan, _requests

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


# ---- the plan, where tokens get no place ----


def _holes(seed, B, page, most, prompts, longest, holes):
    """Requests as a server has them, with `holes` of their pages and of the list's not there."""
    rng = np.random.default_rng(seed)
    have, fresh, table, free, pages = _requests(rng, B, page, most, prompts, longest)
    table[rng.random(table.shape) < holes] = pages
    free = np.where(rng.random(len(free)) < holes, rng.choice([-1, -(1 << 31), pages, (1 << 31) - 1], len(free)), free)
    return have, fresh, table, free, pages, int(fresh.sum())


# one workgroup; several, whose first one counts; the same with pages of one and two tokens, which are counted by a launch of their own; more requests than threads
@pytest.mark.parametrize("holes", [0.0, 0.15, 1.0])
@pytest.mark.parametrize("B,page,most,prompts,longest", [(7, 4, 9, 0.5, 30), (300, 8, 64, 0.3, 60), (300, 8, 64, 0.9, 90), (1, 16, 2000, 1.0, 19999), (1024, 16, 40, 0.5, 100),
                                                         (1000, 1, 200, 0.9, 190), (3, 2, 50000, 1.0, 60000), (1025, 16, 8, 0.2, 30), (2500, 64, 5, 0.2, 100)])
def test_tokens_without_a_place_are_counted(B, page, most, prompts, longest, holes):
    have, fresh, table, free, pages, total = _holes(B, B, page, most, prompts, longest, holes)
    for rows in (total + 5, max(total - total // 9, 0)):
        for part in (len(free), len(free) // 2):
            for in_place in (False, True):
                want = _plan(have, fresh, 0, free[:part], min(3, part), table, pages, page, rows, in_place)
                assert want[5][1] == total - sum(s >= 0 for s in want[3])


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("B,T,page", [(3, 40, 16), (5, 5000, 16), (4, 50000, 1), (1030, 1100, 16)])
def test_counts_stop_at_the_largest_number(B, T, page, in_place):
    """More tokens than 2^31 - 1 are asked for, one fewer, one more; none of them has a place."""
    for total in ((1 << 31) - 2, (1 << 31) - 1, 1 << 31, (1 << 32) + 7):
        first = min(total // 2, (1 << 31) - 1)
        second = min(total - first, (1 << 31) - 1)
        fresh = [first, second, total - first - second] + [0] * (B - 3)
        dev, taken, table = ints(fresh), ints([0, 0]), ints([[-1]] * B)
        counts = taken if in_place else ints([3, 3])
        rows, lengths, slots, positions = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (B + 1, B, T, T))
        nb = L.cgbn_page_plan_workspace_bytes(B, T)
        L.cgbn_page_plan(ints([0] * B), dev, B, 0, ints([0]), 0, taken, counts, table, 1, 4, page, T, rows, lengths, slots, positions, workspace(nb), nb)
        torch.cuda.synchronize()
        assert counts.tolist() == [0, min(total, (1 << 31) - 1)] and bool((slots == -1).all())


def test_steps_after_the_pages_have_ended():
    """A server's steps in a graph: every token that gets no place is counted in its step."""
    B, page, most, pages, T = 4, 4, 9, 6, 8
    have, fresh, taken, table, free = ints([0] * B), ints([0] * B), ints([0, 0]), ints([[-1] * most] * B), ints(range(pages))
    rows, lengths, slots, positions = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (B + 1, B, T, T))

    def step():
        L.cgbn_page_plan(have, fresh, B, 0, free, pages, taken, taken, table, most, pages, page, T, rows, lengths, slots, positions)
        have.copy_(lengths)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lost = []
    for more in ([2, 1, 2, 3], [2, 2, 2, 2], [2, 2, 1, 3], [1, 1, 1, 1], [1, 1, 1, 1], [2, 2, 2, 2], [5, 5, 0, 0]):
        fresh.copy_(ints(more))
        graph.replay()
        torch.cuda.synchronize()
        given = slots.tolist()
        assert taken.tolist()[1] == sum(more) - sum(s >= 0 for s in given)
        lost.append(taken.tolist()[1])
    assert lost[0] == 0 and all(lost[-3:])


def test_a_full_cache_goes_on_counting():
    blk = B.Block(channels=64, heads=2, head_size=32, width=96, positions=128, dtype="f32")
    pages = B.Pages(blk, requests=2, rows=4, pages=2, page=2, most=9)
    x = torch.randn(4, 64, device=DEV)
    pages.fresh.fill_(2)
    pages.step(x)
    for n in range(1, 5):
        pages.fresh.copy_(torch.tensor([1, n % 2]))
        pages.step(x)
        assert pages.taken.tolist() == [2, 1 + n % 2]


def test_steps_of_fewer_rows():
    """Of as many as there are tokens, and of fewer: what is cut off is counted; a captured one goes on beside eager ones of more rows."""
    blk = B.Block(channels=64, heads=2, head_size=32, width=96, positions=512, dtype="bf16")
    x = torch.randn(300, 64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(5)).to(blk.dt)
    eager, captured = (B.Pages(blk, requests=3, rows=300, pages=600, page=4, most=200) for _ in range(2))
    one = x[:3].clone()
    captured.fresh.zero_()
    captured.step(one)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = captured.step(one)
    for n, fresh in enumerate([[1, 1, 1], [100, 50, 150], [1, 1, 1], [1, 0, 1], [290, 1, 3], [1, 1, 1], [2, 2, 2]]):
        for p in (eager, captured):
            p.fresh.copy_(torch.tensor(fresh))
        if sum(fresh) > 6:
            want, got = eager.step(x), captured.step(x)
            blk._linear(x.repeat(40, 1), blk.p["o"])          # (what a workspace was before would be taken by others)
        else:
            one.copy_(x[n:n + 3])
            want, got = eager.step(one), out
            graph.replay()
        torch.cuda.synchronize()
        rows = min(sum(fresh), len(want))
        assert torch.equal(got[:rows], want[:rows]) and torch.equal(captured.table, eager.table) and torch.equal(captured.k, eager.k), n
        assert eager.taken.tolist()[1] == captured.taken.tolist()[1] == sum(fresh) - rows
    # the same rows with padding behind them and without, by other tiles
    results = []
    for rows in (x[:3], x):
        pages = B.Pages(blk, requests=3, rows=300, pages=600, page=4, most=200)
        pages.fresh.fill_(1)
        results.append(pages.step(rows)[:3])
    assert _off(results[0], results[1].cpu()) <= 3e-2
