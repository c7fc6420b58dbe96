"""cgbn_linear_*: every value against the oracle, at the sizes where tiles, steps, splits and chunks end."""

import numpy as np
import pytest
import torch

from layers_harness import DEV, UNIT, F, Linear, f64, near
from paper_1711_07240_amd import cgbn as L

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "silu"]
# M: below, at and beyond the few-rows kernels' blocks and the tiles' edges; N: no whole chunk, a tile's edge; K: shorter than a
# chunk, than a step, no whole chunk (padded copies), ends inside a step
FORWARD = [(1, 1, 1), (1, 1024, 1024), (2, 17, 9), (15, 40, 72), (16, 64, 64), (17, 100, 256), (32, 48, 1000), (33, 64, 64), (40, 8, 8),
           (64, 65, 63), (65, 72, 136), (129, 130, 131), (200, 256, 64), (257, 300, 520), (300, 72, 2056), (513, 264, 24), (70, 1, 4096),
           (1000, 3, 5), (100, 512, 3000), (2100, 520, 72)]
BACKWARD = [(1, 1, 1), (1, 64, 64), (2, 17, 9), (16, 40, 72), (33, 64, 64), (64, 65, 63), (130, 257, 131), (257, 300, 264), (3000, 8, 40),
            (5000, 128, 64), (70, 1, 300), (300, 264, 8), (1025, 72, 520), (9, 2056, 24)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", FORWARD, ids=str)
def test_forward(size, dtype):
    act = ACTS[sum(size) % 4]
    p = Linear(*size, dtype)
    p.check_forward(act)
    p.check_forward("none", bias=False, residual=False, save=False)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forward_activations(act, dtype):
    for size in ((5, 40, 64), (140, 72, 96)):
        p = Linear(*size, dtype, seed=1, scale=3.0)
        for bias, residual, save in ((True, False, False), (False, True, True), (True, True, False)):
            p.check_forward(act, bias, residual, save)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", BACKWARD, ids=str)
def test_backward(size, dtype):
    p = Linear(*size, dtype)
    p.check_backward(ACTS[sum(size) % 4])
    p.check_backward("none")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("want", [("dx",), ("dw",), ("dbias",), ("dresidual",), ("dx", "dw"), ("dw", "dresidual"), ("dx", "dbias")], ids="-".join)
def test_backward_of_what_is_wanted(want, act):
    for size in ((100, 40, 64), (37, 41, 24)):
        Linear(*size, "bf16", seed=2).check_backward(act, want)


def test_in_place():
    p = Linear(70, 64, 96, "bf16")
    y, _ = p.forward("relu", save=False)
    M, N, K = p.size
    r = p.residual.clone()
    ws = torch.empty(L.cgbn_linear_workspace_bytes(M, N, K, "bf16", True), dtype=torch.uint8, device=DEV)
    L.cgbn_linear_forward(p.x, p.w, p.bias, r, M, N, K, "relu", r, None, "bf16", ws)
    assert torch.equal(r, y)
    for act in ("none", "silu"):
        out, _ = p.backward(act)
        dy, dx, dw = p.dy.clone(), torch.empty_like(p.x), torch.empty_like(p.w)
        L.cgbn_linear_backward(dy, p.x, p.w, p.saved, M, N, K, act, dx, dw, None, dy, "bf16", ws)
        assert torch.equal(dy, out["dresidual"]) and torch.equal(dx, out["dx"]) and torch.equal(dw, out["dw"])


def test_no_rows():
    dw, dbias = torch.full((8, 16), 7.0, device=DEV), torch.full((8,), 7.0, device=DEV)
    w, none = torch.ones(8, 16, device=DEV), torch.empty(0, device=DEV)
    L.cgbn_linear_forward(none, w, None, None, 0, 8, 16, "gelu", none)
    L.cgbn_linear_backward(none, none, w, None, 0, 8, 16, "gelu", None, dw, dbias)
    assert not dw.any() and not dbias.any()


def test_infinities_and_nan_stay_in_their_sums():
    """One row of x, one of W and one value of the residual are not finite: the other results do not know."""
    for size in ((20, 40, 70), (200, 72, 200)):
        for dtype in ("bf16", "f32"):
            p = Linear(*size, dtype, seed=3)
            clean, _ = p.forward("none", save=False)
            p.x[3, 5], p.x[7, 0], p.w[9, 2], p.residual[11, 13] = float("inf"), float("nan"), float("-inf"), float("nan")
            got, _ = p.forward("none", save=False)
            touched = torch.zeros_like(got, dtype=torch.bool)
            touched[3], touched[7], touched[:, 9], touched[11, 13] = True, True, True, True
            assert torch.equal(got[~touched], clean[~touched])
            assert not torch.isfinite(got[touched]).any()


def test_relu_passes_no_infinity_where_it_is_closed():
    p = Linear(100, 40, 64, "bf16", seed=4)
    shut = p.saved <= 0
    p.dy[shut] = float("inf")
    out, _ = p.backward("relu")
    assert not out["dresidual"][shut].any() and all(bool(torch.isfinite(t).all()) for t in out.values())


def test_same_bits_every_time_and_on_another_stream():
    for size in ((16, 256, 2048), (300, 264, 2056), (5000, 72, 64)):
        p = Linear(*size, "bf16", seed=5)
        y, z = p.forward("gelu")
        out, _ = p.backward("gelu")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            with torch.cuda.stream(s):
                y2, z2 = p.forward("gelu")
                out2, _ = p.backward("gelu")
            assert torch.equal(y, y2) and torch.equal(z, z2) and all(torch.equal(out[k], out2[k]) for k in out)


def test_graph_replays():
    """The calls captured once; every replay, with the program's own work between, gives what the eager calls give."""
    M, N, K = 300, 264, 2056
    p = Linear(M, N, K, "bf16", seed=6)
    y, _ = p.forward("silu", save=False)
    back, saved = p.backward("silu")
    ws = torch.empty(max(L.cgbn_linear_workspace_bytes(M, N, K, "bf16", b) for b in (False, True)), dtype=torch.uint8, device=DEV)
    o = {k: torch.zeros_like(v) for k, v in back.items()}
    o["y"] = torch.zeros_like(y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.cgbn_linear_forward(p.x, p.w, p.bias, p.residual, M, N, K, "silu", o["y"], None, "bf16", ws)
        L.cgbn_linear_backward(p.dy, p.x, p.w, p.saved, M, N, K, "silu", o["dx"], o["dw"], o["dbias"], o["dresidual"], "bf16", ws)
    for _ in range(4):
        for t in o.values():
            t.fill_(3.0)
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o["y"], y) and all(torch.equal(o[k], back[k]) for k in back)


def _near_product(got, a, b, what):
    want = a @ b
    near(got, want, UNIT["bf16"] * np.abs(want) + (a.shape[1] + 8) * F * (np.abs(a) @ np.abs(b)) * 1.01, what)


def test_rows_beyond_32_bit_offsets():
    """A tall matrix whose last rows lie beyond 2^32 elements; they and the first are compared."""
    M, N, K = (1 << 32) // 1024 + 515, 8, 1024
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(5)
    x[-600:] = torch.randn(600, K, device=DEV, generator=gen).to(torch.bfloat16)
    x[:5] = 1.0
    w = torch.randn(N, K, device=DEV, generator=gen).to(torch.bfloat16)
    y = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(L.cgbn_linear_workspace_bytes(M, N, K, "bf16", True), dtype=torch.uint8, device=DEV)
    L.cgbn_linear_forward(x, w, None, None, M, N, K, "none", y, None, "bf16", ws)
    for rows in (slice(0, 5), slice(M - 600, M)):
        _near_product(y[rows], f64(x[rows]), f64(w).T, "y")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    dy = torch.zeros(M, N, dtype=torch.bfloat16, device=DEV)
    dy[-3:] = 1.0
    L.cgbn_linear_backward(dy, x, w, None, M, N, K, "none", dx, dw, None, None, "bf16", ws)
    _near_product(dx[-4:], f64(dy[-4:]), f64(w), "dx")
    _near_product(dw, f64(dy[-3:]).T, f64(x[-3:]), "dw")
