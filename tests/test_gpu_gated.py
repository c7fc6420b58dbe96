"""cgbn_gated_*: every value against the oracle, at the sizes where tiles, steps, splits and chunks end."""

import pytest
import torch

from layers_harness import DEV, Gated
from paper_1711_07240_amd import cgbn as L

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "silu"]
SIZES = [(1, 1, 1), (1, 256, 512), (3, 17, 9), (16, 40, 72), (17, 33, 130), (33, 32, 64), (64, 65, 63), (130, 129, 131), (257, 300, 264),
         (300, 40, 2056), (1030, 136, 24), (40, 8, 3000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(size, dtype):
    p = Gated(*size, dtype)
    p.check_forward(ACTS[sum(size) % 4])
    p.check_forward("silu", save=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward(size, dtype):
    p = Gated(*size, dtype)
    p.check_backward(ACTS[sum(size) % 4])


@pytest.mark.parametrize("act", ACTS)
def test_activations_and_wanted_outputs(act):
    p = Gated(100, 72, 96, "bf16", seed=1)
    p.check_forward(act)
    p.check_backward(act, dw=False)
    p.check_backward(act, dx=False)


def test_no_rows():
    dwg, dwu, none = torch.full((8, 16), 7.0, device=DEV), torch.full((8, 16), 7.0, device=DEV), torch.empty(0, device=DEV)
    w = torch.ones(8, 16, device=DEV)
    L.cgbn_gated_forward(none, w, w, 0, 8, 16, "silu", none)
    L.cgbn_gated_backward(none, none, w, w, none, none, 0, 8, 16, "silu", None, dwg, dwu)
    assert not dwg.any() and not dwu.any()


def test_nan_stays_in_its_sums():
    for size in ((20, 40, 72), (200, 72, 200)):
        p = Gated(*size, "bf16", seed=2)
        run = lambda: _forward(p)
        clean = run()
        p.x[3, 5], p.wu[9, 2] = float("nan"), float("inf")
        got = run()
        touched = torch.zeros_like(got, dtype=torch.bool)
        touched[3], touched[:, 9] = True, True
        assert torch.equal(got[~touched], clean[~touched])


def _forward(p):
    M, F, K = p.size
    h = torch.empty(M, F, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(L.cgbn_gated_workspace_bytes(M, F, K, p.dtype, False), dtype=torch.uint8, device=DEV)
    L.cgbn_gated_forward(p.x, p.wg, p.wu, M, F, K, "silu", h, None, None, p.dtype, ws)
    return h


def test_same_bits_every_time():
    for size in ((4, 264, 2048), (300, 264, 2056)):
        p = Gated(*size, "bf16", seed=3)
        first = _forward(p)
        for _ in range(4):
            assert torch.equal(first, _forward(p))
