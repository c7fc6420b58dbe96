"""The rotation by scaled positions, the plan of a paged cache and its store against their definitions."""

import numpy as np
import pytest
import torch

from layers_harness import DEV, F, TORCH, UNIT, check_guard, f64, near, normal, workspace
from oracle import serving_oracle as V
from paper_1711_07240_amd import cgbn as L
from serving_harness import ints

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16"]


# ---- rotation ----


def _frequencies(R, *scaling):
    f = torch.empty(R // 2, dtype=torch.float64)
    L.cgbn_rotary_frequencies(R, 10000.0, *(scaling or ("none", 1.0, 0.0, 0.0, 0.0)), f)
    return f


class Turned:
    def __init__(self, T, Hq, Hk, D, R, dtype, far=4096, gap=0, shift=0, magnitude=1.0, seed=0):
        rng = np.random.default_rng(seed + T + 7 * D + R)
        self.size, self.R, self.dtype, self.magnitude = (T, Hq, Hk, D), R, dtype, magnitude
        self.row = (Hq + 2 * Hk) * D + gap
        flat = normal(rng, T * self.row + shift, dtype=dtype)
        self.qkv = flat[shift:].view(T, self.row)
        self.q, self.k = self.qkv[:, :Hq * D], self.qkv[:, Hq * D:(Hq + Hk) * D]
        self.positions = ints(rng.integers(-far // 8, far, T))
        self.freq = _frequencies(R, "parts", 8.0, 4096.0, 32.0, 1.0).to(DEV)

    def check(self, style, back=False, in_place=False, positions=True):
        T, Hq, Hk, D = self.size
        at = f64(self.positions) if positions else np.arange(T)
        fn = L.cgbn_rotate_backward if back else L.cgbn_rotate_forward
        q0, k0 = f64(self.q), f64(self.k)
        if in_place:
            data = self.qkv.clone()
            yq, yk, ld = data[:, :Hq * D], data[:, Hq * D:(Hq + Hk) * D], (self.row, self.row)
            xq, xk = yq, yk
        else:
            data = torch.full((T, (Hq + Hk) * D + 24), 7.0, dtype=TORCH[self.dtype], device=DEV)
            yq, yk, ld = data[:, 8:8 + Hq * D], data[:, 16 + Hq * D:16 + (Hq + Hk) * D], (data.shape[1],) * 2
            xq, xk = self.q, self.k
        fn(xq, self.row, xk, self.row, T, Hq, Hk, D, self.R, style, self.positions if positions else None, self.freq, self.magnitude, yq, ld[0], yk, ld[1],
           self.dtype)
        torch.cuda.synchronize()
        for name, got, x, heads in (("q", yq, q0, Hq), ("k", yk, k0, Hk)):
            if not heads:
                continue
            want = V.rotate(x, heads, D, self.R, style, at, f64(self.freq), self.magnitude, back)
            size = V.rotate(np.abs(x), heads, D, self.R, style, np.zeros(T), f64(self.freq), 1.0)
            first = np.abs(size.reshape(T, heads, D))
            pair = first.copy()
            if self.R:
                i = np.arange(self.R // 2) if style == "halves" else np.arange(0, self.R, 2)
                j = i + (self.R // 2 if style == "halves" else 1)
                pair[..., i] = pair[..., j] = self.magnitude * (first[..., i] + first[..., j])
            # cosine and sine are off by at most 4 units of 1 (the rest of the angle, the polynomial, the magnitude), products and the sum by 2 each; the angle
            # in 64 bits by 2^-52 of itself
            err = (8 * F + 2.0 ** -52 * np.abs(at).max()) * pair.reshape(T, -1)
            err[:, np.tile(np.arange(D) >= self.R, heads)] = 0          # those that are not turned are copied
            near(got, want, err + UNIT[self.dtype] * np.abs(want) * (np.tile(np.arange(D) < self.R, heads)) + 1e-37, f"{name} {self.size} {self.R} {style}")
        if not in_place:
            assert bool((data[:, :8] == 7.0).all()) and bool((data[:, -8:] == 7.0).all())
        else:
            assert torch.equal(data[:, (Hq + Hk) * D:], self.qkv[:, (Hq + Hk) * D:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("style", ["halves", "interleaved"])
@pytest.mark.parametrize("size", [(1, 1, 1, 8, 8), (3, 2, 1, 64, 64), (5, 4, 4, 80, 32), (7, 6, 2, 128, 20), (9, 3, 0, 96, 96), (2, 1, 1, 1024, 1024),
                                  (4, 2, 2, 39, 38), (3, 5, 1, 66, 12), (6, 2, 2, 16, 0), (300, 40, 8, 128, 128), (2, 1, 1, 33, 2), (130, 1, 1, 2, 2)], ids=str)
def test_rotation(size, style, dtype):
    T, Hq, Hk, D, R = size
    a = Turned(T, Hq, Hk, D, R, dtype, magnitude=1.25)
    for back in (False, True):
        a.check(style, back)
        a.check(style, back, in_place=True)
    a.check(style, positions=False)


@pytest.mark.parametrize("dtype", TYPES)
def test_rotation_of_rows_on_odd_places(dtype):
    for gap, shift in ((1, 0), (0, 1), (2, 2), (4, 4), (3, 5)):
        for style in ("halves", "interleaved"):
            Turned(11, 3, 2, 48, 24, dtype, gap=gap, shift=shift).check(style)
            Turned(11, 3, 2, 48, 24, dtype, gap=gap, shift=shift).check(style, back=True, in_place=True)


@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 1])
def test_rotation_of_far_positions(far):
    Turned(200, 2, 1, 64, 64, "f32", far=far).check("halves")


def test_large_rotation_goes_past_the_caches():
    Turned(9001, 12, 4, 128, 128, "bf16", far=200000).check("halves")
    Turned(5003, 12, 4, 96, 32, "f32", far=200000).check("interleaved", back=True)


@pytest.mark.parametrize("style", ["halves", "interleaved"])
def test_rotation_backward_is_the_gradient(style):
    """Of <dy, rotate(x)>: by differences of the forward pass, which is linear, so that a difference of any size is exact up to rounding."""
    T, H, D, R = 3, 2, 16, 12
    a = Turned(T, H, 0, D, R, "f32", magnitude=1.5)
    dy = normal(np.random.default_rng(1), T, H * D)
    dq = torch.empty_like(dy)
    L.cgbn_rotate_backward(dy, H * D, None, 0, T, H, 0, D, R, style, a.positions, a.freq, a.magnitude, dq, H * D, None, 0)
    y0, y1 = (torch.empty_like(dy) for _ in range(2))
    x = a.q.contiguous()
    for t, d in ((0, 0), (1, 7), (2, 11), (2, 12), (0, 31), (1, 16)):
        step = torch.zeros_like(x)
        step[t, d] = 2.0
        for y, z in ((y0, x - step), (y1, x + step)):
            L.cgbn_rotate_forward(z, H * D, None, 0, T, H, 0, D, R, style, a.positions, a.freq, a.magnitude, y, H * D, None, 0)
        numeric = float((f64(dy) * (f64(y1) - f64(y0))).sum() / 4)
        # four values of size up to 8 a row, each rounded a few times, times dy of up to 4
        assert abs(numeric - f64(dq)[t, d]) <= 64 * 8 * 4 * F


def test_values_that_are_not_turned_keep_what_they_hold():
    x = torch.full((2, 24), float("inf"), device=DEV)
    x[:, :10] = 1.0
    y = torch.empty_like(x)
    for style in ("halves", "interleaved"):
        L.cgbn_rotate_forward(x, 24, None, 0, 2, 1, 0, 24, 10, style, None, _frequencies(10).to(DEV), 1.0, y, 24, None, 0)
        assert bool(torch.isinf(y[:, 10:]).all()) and bool(torch.isfinite(y[:, :10]).all())


# ---- plan ----


def _plan(have, fresh, before, free, taken, table, pages, page, T, in_place=False):
    B, most = len(have), len(table[0]) if len(table) else 1
    dev = [ints(x) for x in (have, fresh, free if len(free) else [0])]
    tab = ints(table) if B else ints([[0]])
    taken_dev = ints([taken, 77])
    counts = taken_dev if in_place else ints([5, 5])
    out = [torch.full((n + 3,), 99, dtype=torch.int32, device=DEV) for n in (B + 1, B, T, T)]
    nb = L.cgbn_page_plan_workspace_bytes(B, T)
    ws = workspace(nb)
    L.cgbn_page_plan(dev[0], dev[1], B, before, dev[2], len(free), taken_dev, counts, tab, most, pages, page, T, *out, ws, nb)
    torch.cuda.synchronize()
    check_guard(ws, nb)
    want = V.plan(have, fresh, before, free, taken, table, most, pages, page, T)
    for name, got, ref in zip(("rows", "lengths", "slots", "positions"), out, (want[0], want[1], want[3], want[4])):
        got = got.cpu().numpy()
        assert (got[-3:] == 99).all(), name
        assert np.array_equal(got[:-3], np.asarray(ref, np.int64)), name
    if B:
        assert np.array_equal(tab.cpu().numpy(), want[2])
    assert counts[:2].cpu().tolist() == want[5]
    return want


def _requests(rng, B, page, most, prompts, longest):
    have = rng.integers(0, most * page // 2 + 1, B)
    fresh = np.where(rng.random(B) < prompts, rng.integers(0, longest + 1, B), 1)
    held = -(-have // page)
    order = rng.permutation(int(held.sum() + (fresh // page + 2).sum()))
    table = np.full((B, most), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    return have, fresh, table, order[at:], len(order)


@pytest.mark.parametrize("B,T,page,most,prompts,longest", [(1, 1, 16, 4, 0.0, 1), (7, 7, 1, 9, 0.0, 1), (16, 40, 16, 30, 0.5, 9), (300, 4096, 8, 64, 0.3, 60),
                                                           (1024, 1024, 32, 16, 0.0, 1), (300, 5000, 8, 64, 0.3, 60), (1025, 1100, 16, 8, 0.0, 1),
                                                           (2500, 9001, 64, 5, 0.2, 100), (1, 20000, 16, 2000, 1.0, 19999), (3, 4097, 1024, 3, 1.0, 2000)])
def test_plans(B, T, page, most, prompts, longest):
    rng = np.random.default_rng(B + T)
    have, fresh, table, free, pages = _requests(rng, B, page, most, prompts, longest)
    taken = min(3, len(free))
    _plan(have, fresh, 1000, free, taken, table, pages, page, T)
    _plan(have, fresh, 0, free, taken, table, pages, page, T, in_place=True)
    # as many rows as there are, one fewer, and a list that ends in between
    total = int(fresh.sum())
    for rows in (total, max(total - 1, 0), total // 2):
        _plan(have, fresh, 0, free[:len(free) // 2], taken, table, pages, page, rows)


def test_plans_of_nothing_and_of_nonsense():
    assert _plan([], [], 0, [3, 4], 1, [], 8, 16, 5)[0] == [0]
    _plan([0], [0], 7, [], 0, [[-1, -1]], 4, 16, 3)
    _plan([0], [4], 7, [], 0, [[-1, -1]], 4, 16, 4)
    # less than nothing, more than the table holds, pages that are not there, a count beyond the list
    table = [[2, 9, -1], [-7, 1, 1 << 30], [0, 1, 2], [5, 5, 5]]
    _plan([-5, 17, 1000, 48], [3, 40, 2, 1], 0, [9, 8, -1, 1 << 30, 3], 0, table, 9, 16, 60)
    _plan([-5, 17, 1000, 48], [3, 40, 2, 1], 0, [9, 8, 3], 50, table, 10, 16, 60)
    _plan([-5, 17, 10, 2], [3, 40, -2, 2 ** 31 - 1], 0, list(range(9)), 1, table, 10, 16, 5000)
    _plan([0, 0, 0, 0], [2 ** 31 - 1] * 4, 0, list(range(9)), 1, table, 10, 16, 100)


def test_steps_of_requests_that_grow():
    """Step after step on the device, in one captured graph: what a step leaves is what the next begins with, and every page is somebody's alone."""
    B, page, most, pages, T = 5, 4, 6, 40, 12
    rng = np.random.default_rng(0)
    free = rng.permutation(pages)
    have, fresh, taken, table = ints([0] * B), ints([1] * B), ints([0, 0]), ints([[-1] * most] * B)
    rows, lengths, slots, positions = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (B + 1, B, T, T))
    free_dev = ints(free)

    def step():
        L.cgbn_page_plan(have, fresh, B, 0, free_dev, pages, taken, taken, table, most, pages, page, T, rows, lengths, slots, positions)
        have.copy_(lengths)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    h, t, tab, seen = [0] * B, 0, [[-1] * most] * B, set()
    for n in range(9):
        more = rng.integers(0, 4, B)
        fresh.copy_(ints(more))
        graph.replay()
        torch.cuda.synchronize()
        want = V.plan(h, more, 0, free, t, tab, most, pages, page, T)
        for got, ref in zip((rows, lengths, table, slots, positions, taken), want):
            assert np.array_equal(got.cpu().numpy(), np.asarray(ref)), n
        h, tab, t = want[1], want[2], want[5][0]
        places = [s for s in slots.cpu().tolist() if s >= 0]
        assert len(places) == len(set(places)) and not seen & set(places)
        seen |= set(places)


# ---- store ----


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Hk,D,page", [(1, 1, 8, 1), (5, 8, 128, 16), (77, 3, 40, 8), (1000, 20, 80, 32), (3, 64, 256, 4), (300, 1, 16, 1024)])
def test_store(T, Hk, D, page, dtype):
    rng = np.random.default_rng(T + D)
    pages = 2 * T // page + 3
    slots = rng.permutation(pages * page)[:T]
    slots[rng.random(T) < 0.1] = -1
    if T > 4:
        slots[1], slots[3] = pages * page, -(1 << 31)
    kv = normal(rng, T, 2 * Hk * D + 8, dtype=dtype)
    k, v = kv[:, :Hk * D], kv[:, Hk * D:2 * Hk * D]
    pools = [normal(rng, pages, Hk, page, D, dtype=dtype) for _ in range(2)]
    want = [V.store(f64(x), Hk, D, slots, f64(p)) for x, p in zip((k, v), pools)]
    L.cgbn_page_store(k, kv.shape[1], v, kv.shape[1], T, Hk, D, ints(slots), *pools, pages, page, dtype)
    torch.cuda.synchronize()
    for p, w in zip(pools, want):
        assert np.array_equal(f64(p), w)


def test_store_keeps_every_bit():
    x = torch.tensor([[0x7fc1, 0x7f81, 0xffff, 0x8000, 0x0001, 0x7f80, 0xff80, 0x3f80]], dtype=torch.int32).to(torch.int16).to(DEV)
    pools = [torch.zeros(2, 1, 4, 8, dtype=torch.int16, device=DEV) for _ in range(2)]
    L.cgbn_page_store(x, 8, x.clone(), 8, 1, 1, 8, ints([6]), *pools, 2, 4, "bf16")
    for p in pools:
        assert torch.equal(p[1, 0, 2], x[0]) and int((p != 0).sum()) == int((x != 0).sum())
