"""The layers beside the normalization on the ways that only some sizes take: long reductions of few rows, which workgroups share; some dozen
rows with large weights; dx split beside the other product of its launch; results that go past the caches; rows that go in 8 bytes and not
in 16.  Then what float products keep of their operands, and gradients against differences of the forward pass."""

import numpy as np
import pytest
import torch

from layers_harness import ACT_ERR, DEV, F, STEEP, UNIT, Gated, Linear, f64, near, normal
from oracle import layers_oracle as Y
from paper_1711_07240_amd import cgbn as L
from test_gpu_head_norm import Heads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size,dtype", [((1, 64, 8192), "bf16"), ((2, 1024, 8192), "bf16"), ((16, 40, 12300), "bf16"), ((5, 33, 8191), "bf16"),
                                        ((20, 50, 9000), "bf16"), ((32, 16, 6145), "bf16"), ((3, 64, 4000), "f32"), ((16, 7, 12289), "f32"),
                                        ((25, 90, 4001), "f32")], ids=str)
def test_few_rows_of_a_long_reduction(size, dtype):
    p = Linear(*size, dtype)
    p.check_forward("gelu")
    p.check_forward("none", bias=False, residual=False, save=False)


@pytest.mark.parametrize("size,dtype", [((1, 64, 8192), "bf16"), ((16, 33, 6200), "bf16"), ((4, 48, 8191), "bf16"), ((2, 64, 5248), "f32"),
                                        ((16, 20, 4001), "f32")], ids=str)
def test_few_rows_of_a_long_gated_reduction(size, dtype):
    p = Gated(*size, dtype)
    p.check_forward("silu")
    p.check_forward("gelu", save=False)


@pytest.mark.parametrize("size", [(1, 1, 65), (1, 17, 127), (3, 33, 1025), (8, 40, 4069), (16, 50, 2113), (17, 100, 1001), (32, 31, 4097), (2, 16, 8193)], ids=str)
def test_few_rows_of_odd_length(size):
    Linear(*size, "bf16").check_forward("silu")
    p = Linear(*size, "bf16", seed=1)
    p.check_forward("none", bias=False, residual=False, save=False)
    Gated(*size, "bf16").check_forward("gelu")


@pytest.mark.parametrize("size,dtype", [((17, 8192, 4096), "bf16"), ((31, 6000, 4104), "bf16"), ((32, 4097, 4100), "bf16"), ((32, 8192, 4096), "f32")],
                         ids=str)
def test_some_rows_with_large_weights(size, dtype):
    Linear(*size, dtype).check_forward("relu")


@pytest.mark.parametrize("size,dtype", [((64, 4096, 512), "bf16"), ((64, 4096, 512), "f32"), ((160, 5461, 130), "bf16"), ((250, 2560, 70), "f32"),
                                        ((33, 8192, 64), "bf16")], ids=str)
def test_backward_of_wide_results_and_some_rows(size, dtype):
    Linear(*size, dtype).check_backward("silu")
    Gated(*size, dtype).check_backward("silu")


@pytest.mark.parametrize("size,dtype", [((16500, 1024, 40), "bf16"), ((4100, 4099, 24), "bf16"), ((40000, 500, 9), "bf16"), ((2100, 4097, 16), "f32")],
                         ids=str)
def test_large_results(size, dtype):
    Linear(*size, dtype).check_forward("gelu")


@pytest.mark.parametrize("size,dtype", [((40000, 24, 512), "bf16"), ((16700, 17, 1031), "bf16"), ((12000, 16, 700), "f32")], ids=str)
def test_large_gradients(size, dtype):
    Linear(*size, dtype).check_backward("relu")


@pytest.mark.parametrize("size,dtype", [((4100, 4100, 40), "bf16"), ((8300, 2051, 24), "bf16"), ((2100, 4097, 16), "f32")], ids=str)
def test_large_gated_results(size, dtype):
    Gated(*size, dtype).check_forward("silu")


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("size", [(196700, 256, 40), (98400, 512, 129), (131100, 330, 513), (12389, 4096, 64), (66000, 767, 1000)], ids=str)
def test_many_tiles_and_a_short_reduction(size, residual):
    M, N, K = size
    gen = torch.Generator(device=DEV).manual_seed(K)
    x, w = (torch.randn(r, K, device=DEV, generator=gen).to(torch.bfloat16) for r in (M, N))
    bias, res = torch.randn(N, device=DEV, generator=gen), torch.randn(M, N, device=DEV, generator=gen).to(torch.bfloat16)
    y, z = (torch.full((M + 1, N), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ws = torch.empty(L.cgbn_linear_workspace_bytes(M, N, K, "bf16", False), dtype=torch.uint8, device=DEV)
    L.cgbn_linear_forward(x, w, bias, res if residual else None, M, N, K, "gelu", y, z, "bf16", ws)
    assert bool((y[M] == 7.0).all()) and bool((z[M] == 7.0).all())
    # some rows exactly, the edges among them; every row against a product in float on the device, twice as far off at most
    rows = torch.unique(torch.cat([torch.arange(200), torch.arange(M - 200, M), torch.randint(0, M, (600,), generator=torch.Generator().manual_seed(1))]))
    xs, ws64, b, r = f64(x[rows.to(DEV)]), f64(w), f64(bias), f64(res[rows.to(DEV)]) if residual else 0.0
    want = Y.linear_forward(xs, ws64, b, r if residual else None, "gelu")
    err = (K + 8) * F * (np.abs(xs) @ np.abs(ws64).T + np.abs(b) + np.abs(r))
    u = UNIT["bf16"]
    near(z[rows.to(DEV)], want[1], err + u * np.abs(want[1]) + 1e-37, "z")
    near(y[rows.to(DEV)], want[0], STEEP * err * (1 + u) + u * np.abs(want[0]) + ACT_ERR * (1 + np.abs(want[1])) + 1e-37, "y")
    wf = w.float().t().contiguous()
    for at in range(0, M, 8192):
        to = min(M, at + 8192)
        full = x[at:to].float() @ wf + bias + (res[at:to].float() if residual else 0.0)
        tol = 2 * (K + 8) * F * (x[at:to].float().abs() @ wf.abs() + bias.abs() + (res[at:to].float().abs() if residual else 0.0)) + u * full.abs()
        assert bool(((z[at:to].float() - full).abs() <= tol).all()), at


@pytest.mark.parametrize("style", ["halves", "interleaved"])
@pytest.mark.parametrize("shape,lead,gap", [((50, 3, 2, 80, 40), 0, 0), ((50, 3, 2, 64, 32), 4, 0), ((50, 3, 2, 64, 32), 0, 4), ((40, 2, 1, 12, 8), 0, 0),
                                            ((40, 2, 1, 100, 24), 0, 0), ((9, 1, 1, 1020, 1000), 0, 0)], ids=str)
def test_rows_in_chunks_of_8_bytes(shape, lead, gap, style):
    p = Heads(*shape, style, "bf16", lead, gap)
    p.check_forward()
    p.check_backward()


@pytest.mark.parametrize("style", ["halves", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape,lead,gap", [((60, 5, 3, 39, 0), 0, 0), ((60, 5, 3, 39, 38), 0, 0), ((60, 5, 3, 39, 20), 1, 0), ((40, 9, 2, 82, 40), 0, 0), ((40, 9, 2, 82, 42), 2, 4),
                                            ((33, 3, 1, 127, 126), 0, 0), ((33, 3, 1, 128, 2), 3, 0), ((17, 3, 1, 129, 128), 0, 0), ((17, 3, 1, 254, 250), 0, 2),
                                            ((9, 40, 2, 3, 2), 0, 0), ((5000, 2, 1, 33, 32), 0, 0), ((1, 1, 1, 35, 34), 0, 0)], ids=str)
def test_rows_in_chunks_of_two_values_and_of_one(shape, lead, gap, dtype, style):
    p = Heads(*shape, style, dtype, lead, gap)
    p.check_forward()
    p.check_backward()


@pytest.mark.parametrize("shape", [(40, 6, 2, 39, 38), (40, 6, 2, 82, 40)], ids=str)
def test_odd_heads_in_place_and_outside_the_table(shape):
    for style in ("halves", "interleaved"):
        p = Heads(*shape, style, "bf16")
        y, (dx, dwq, dwk) = p.forward(), p.backward()
        p.pos[3], p.pos[7] = -1, p.cos.shape[0]
        bad = p.forward()[:, :p.nq + p.nk].view(40, 8, p.D)
        assert not torch.isfinite(bad[[3, 7], :, :p.R]).any() and torch.equal(bad[:3], y[:3, :p.nq + p.nk].view(3, 8, p.D))
        assert torch.equal(bad[3, :, p.R:], y[3, :p.nq + p.nk].view(8, p.D)[:, p.R:])
        p = Heads(*shape, style, "bf16")
        keep = p.x.clone()
        assert torch.equal(p.forward(out=p.x)[:, :p.nq + p.nk], y[:, :p.nq + p.nk])
        p.x.copy_(keep)
        got, gq, gk = p.backward(dx=p.dy)
        assert torch.equal(got[:, :p.nq + p.nk], dx[:, :p.nq + p.nk]) and torch.equal(gq, dwq) and torch.equal(gk, dwk)


@pytest.mark.parametrize("shape,dtype", [((2000, 40, 32, 128, 64), "bf16"), ((1100, 70, 2, 256, 256), "bf16"), ((3000, 30, 6, 80, 32), "f32"),
                                         ((3001, 70, 2, 80, 40), "bf16")], ids=str)
def test_large_norms(shape, dtype):
    p = Heads(*shape, "halves", dtype)
    p.check_forward()
    p.check_backward()


def test_float_products_keep_every_bit():
    """x times the identity is x: nothing of an operand's 24 bits is lost on its way through the matrix cores."""
    for M, K in ((7, 200), (150, 256)):
        rng = np.random.default_rng(M)
        x = torch.from_numpy((rng.standard_normal((M, K)) * 10.0 ** rng.integers(-25, 25, (M, K))).astype(np.float32)).to(DEV)
        eye, y = torch.eye(K, device=DEV), torch.empty(M, K, device=DEV)
        ws = torch.empty(max(L.cgbn_linear_workspace_bytes(M, K, K, "f32", b) for b in (False, True)), dtype=torch.uint8, device=DEV)
        L.cgbn_linear_forward(x, eye, None, None, M, K, K, "none", y, None, "f32", ws)
        assert torch.equal(y, x)
        dx, dw = torch.empty_like(x), torch.empty_like(eye)
        L.cgbn_linear_backward(x, x, eye, None, M, K, K, "none", dx, dw, None, None, "f32", ws)
        assert torch.equal(dx, x)


# Gradients against differences, in float.  Along the unit direction g / |g| of a gradient g the loss sum(dy * y) climbs by |g|.  Four points,
# h = 1/16:  (8 (L(h) - L(-h)) - (L(2h) - L(-2h))) / 12h, off by h^4 / 30 of the fifth derivative, which is bounded below 100 sum|dy| for these
# smooth functions of values near 1 (h^4 / 30 * 100 = 5e-5), and by 1.5 / h of a loss's rounding, (n + 32) 2^-24 sum|dy * y|, n products to a sum.
H = 1.0 / 16


def _climb(loss, tensor, grad):
    norm = float(grad.double().norm())
    start, way = tensor.clone(), grad.double() / norm
    at = {}
    for k in (-2, -1, 1, 2):
        tensor.copy_((start.double() + k * H * way).float())
        at[k] = loss()
    tensor.copy_(start)
    return (8 * (at[1] - at[-1]) - (at[2] - at[-2])) / (12 * H), norm


def _check(loss, pairs, n, dy, y):
    size = float(dy.double().abs().sum())
    tol = 5e-5 * size + 1.5 / H * (n + 32) * F * float((dy.double().abs() * (1 + y.double().abs())).sum())
    for name, tensor, grad in pairs:
        got, want = _climb(loss, tensor, grad)
        assert abs(got - want) <= tol < 0.1 * want, (name, got, want, tol)


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_linear_gradients_against_differences(act):
    M, N, K = 3, 5, 8
    p = Linear(M, N, K, "f32", seed=9)
    y, z = torch.empty(M, N, device=DEV), torch.empty(M, N, device=DEV)
    ws = torch.empty(max(L.cgbn_linear_workspace_bytes(M, N, K, "f32", b) for b in (False, True)) + 16, dtype=torch.uint8, device=DEV)

    def loss():
        L.cgbn_linear_forward(p.x, p.w, p.bias, p.residual, M, N, K, act, y, z, "f32", ws)
        return float((p.dy.double() * y.double()).sum())

    loss()
    dx, dw, db, dr = torch.empty_like(p.x), torch.empty_like(p.w), torch.empty_like(p.bias), torch.empty_like(y)
    L.cgbn_linear_backward(p.dy, p.x, p.w, None if act == "none" else z, M, N, K, act, dx, dw, db, dr, "f32", ws)
    _check(loss, [("x", p.x, dx), ("w", p.w, dw), ("bias", p.bias, db), ("residual", p.residual, dr)], K, p.dy, y)


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_gated_gradients_against_differences(act):
    M, N, K = 3, 5, 8
    rng = np.random.default_rng(4)
    x, wg, wu, dh = normal(rng, M, K), normal(rng, N, K, scale=K ** -0.5), normal(rng, N, K, scale=K ** -0.5), normal(rng, M, N)
    h, gate, up = (torch.empty(M, N, device=DEV) for _ in range(3))
    ws = torch.empty(max(L.cgbn_gated_workspace_bytes(M, N, K, "f32", b) for b in (False, True)) + 16, dtype=torch.uint8, device=DEV)

    def loss():
        L.cgbn_gated_forward(x, wg, wu, M, N, K, act, h, gate, up, "f32", ws)
        return float((dh.double() * h.double()).sum())

    loss()
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    L.cgbn_gated_backward(dh, x, wg, wu, gate, up, M, N, K, act, dx, dwg, dwu, "f32", ws)
    _check(loss, [("x", x, dx), ("gate", wg, dwg), ("up", wu, dwu)], K, dh, h)


@pytest.mark.parametrize("style", ["halves", "interleaved"])
def test_norm_gradients_against_differences(style):
    p = Heads(3, 2, 1, 16, 8, style, "f32", seed=3)
    y = torch.empty_like(p.x)

    def loss():
        p.forward(y)
        return float((p.dy.double() * y.double()).sum())

    loss()
    dx, dwq, dwk = p.backward()
    _check(loss, [("x", p.x, dx), ("wq", p.wq, dwq), ("wk", p.wk, dwk)], 16, p.dy, y)


@pytest.mark.parametrize("size", [(98400, 512, 64), (66000, 767, 1000), (16500, 1024, 40), (20, 1000, 8191)], ids=str)
def test_results_over_the_residual(size):
    """y may be the residual's own buffer: the same bits as elsewhere, and the same in every run."""
    M, N, K = size
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, w, res = (torch.randn(a, b, device=DEV, generator=gen).to(torch.bfloat16) for a, b in ((M, K), (N, K), (M, N)))
    ws = torch.empty(L.cgbn_linear_workspace_bytes(M, N, K, "bf16", False), dtype=torch.uint8, device=DEV)
    y = torch.empty_like(res)
    L.cgbn_linear_forward(x, w, None, res, M, N, K, "relu", y, None, "bf16", ws)
    for _ in range(3):
        over = res.clone()
        L.cgbn_linear_forward(x, w, None, over, M, N, K, "relu", over, None, "bf16", ws)
        assert torch.equal(over, y)


def test_graph_replays_of_shared_and_padded_work():
    """Few rows of a long odd reduction, padded operands, dx split beside dW, odd heads: captured once, replayed with other work between."""
    calls, outs = [], []
    gen = torch.Generator(device=DEV).manual_seed(8)
    rand = lambda *s: torch.randn(*s, device=DEV, generator=gen).to(torch.bfloat16)
    for M, N, K in ((3, 64, 4069), (300, 264, 131), (64, 2048, 512)):
        x, w, dy, b = rand(M, K), rand(N, K), rand(M, N), torch.randn(N, device=DEV, generator=gen)
        y, z, dx, dw, db = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        ws = torch.empty(max(L.cgbn_linear_workspace_bytes(M, N, K, "bf16", k) for k in (False, True)), dtype=torch.uint8, device=DEV)
        calls.append(lambda M=M, N=N, K=K, x=x, w=w, dy=dy, b=b, y=y, z=z, dx=dx, dw=dw, db=db, ws=ws: (
            L.cgbn_linear_forward(x, w, b, None, M, N, K, "silu", y, z, "bf16", ws),
            L.cgbn_linear_backward(dy, x, w, z, M, N, K, "silu", dx, dw, db, None, "bf16", ws)))
        outs += [y, z, dx, dw, db]
    p = Heads(40, 5, 3, 39, 38, "halves", "bf16")
    heads = torch.zeros_like(p.x)
    (q, k), (yq, yk) = p.split(p.x), p.split(heads)
    calls.append(lambda: L.cgbn_head_norm_forward(q, p.row, k, p.row, p.T, p.Hq, p.Hk, p.D, *p.turn(), p.wq, p.wk, 1e-5, yq, p.row, yk, p.row, "bf16"))
    outs.append(heads)
    for call in calls:
        call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for call in calls:
            call()
    for _ in range(4):
        for t in outs[:-1]:
            t.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
