"""Refusals of the layers' entry points beyond those of test_layers_abi.py: buffers that are also another argument's, sizes, workspaces.
Without a GPU: a call that is refused never gets to one."""

import pytest
import torch

from paper_1711_07240_amd import cgbn as L
from test_layers_abi import CALLS, P, _code

# (a call that is wrongly taken would follow addresses that are none)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU")


def _refused(fn, changes, status):
    for change in changes:
        kw = {**CALLS[fn], **change}
        assert _code(fn, kw) == status, (fn, change)
        assert getattr(L.lib(), fn)(*kw.values()) == status, (fn, change)


# the tables' and weights' addresses apart from the tensors'
APART = dict(positions=20 * P, cos=21 * P, sin=22 * P, wq=23 * P, wk=24 * P)


def test_head_norm_results_over_the_other_heads_inputs_or_constants():
    """Queries' results over keys that are still to be read, and the other way; results over the tables."""
    fwd = [{"yq": 2 * P}, {"yk": P}, {"yk": P, "ldyk": 64}, {"yq": 2 * P, "ldyq": 64}]
    fwd += [{**APART, name: P * at} for name in ("yq", "yk") for at in (20, 21, 22, 23, 24)]
    _refused("cgbn_head_norm_forward", fwd, 11)
    bwd = [{"dq": 2 * P}, {"dq": 4 * P}, {"dk": P}, {"dk": 3 * P}, {"dwq": 5 * P}, {"dwk": 6 * P}, {"dwq": 6 * P}, {"dwk": 5 * P}]
    bwd += [{**APART, name: P * at} for name in ("dq", "dk") for at in (20, 21, 22, 23, 24)]
    _refused("cgbn_head_norm_backward", bwd, 11)


def test_head_norm_takes_what_is_not_wrong():
    """In place each over its own, and addresses of what is not read: these calls are refused for their workspace alone, the last thing that is looked
    at."""
    back = {**CALLS["cgbn_head_norm_backward"], **APART, "dwq": 25 * P, "dwk": 26 * P, "workspace_bytes": 0}
    for change in ({}, {"dq": P, "dk": 2 * P, "lddk": 32}, {"dq": 3 * P}, {"Hk": 0, "dq": 2 * P}, {"Hk": 0, "dq": 4 * P}, {"Hk": 0, "dq": 24 * P},
                   {"R": 0, "dq": 21 * P}, {"dk": 4 * P, "lddk": 64}, {"T": 0, "dq": 2 * P}):
        assert _code("cgbn_head_norm_backward", {**back, **change}) == 6, change


def test_more_tiles_than_a_launch_has():
    """Sizes of which no tile shape fits a launch (2^30 rows of 200 floats and more): refused, not done in part."""
    assert L.cgbn_linear_workspace_bytes(1 << 30, 200, 8, "f32", False) == 0
    assert L.cgbn_gated_workspace_bytes(1 << 30, 200, 8, "f32", False) == 0
    big = {"M": 1 << 30, "K": 8, "dtype": 0}
    _refused("cgbn_linear_forward", [{**big, "N": 200}], 2)
    _refused("cgbn_gated_forward", [{**big, "F": 200}], 2)
    # as tall, with a shape that does
    assert L.cgbn_linear_workspace_bytes(1 << 30, 200, 8, "bf16", False) and L.cgbn_linear_workspace_bytes(1 << 30, 128, 8, "f32", False)


def test_a_workspace_that_is_asked_for_is_more_than_256_bytes():
    """Sizes up to 256 say that a call may go without one: a call that refuses to was answered with more."""
    seen = 0
    for dtype in ("f32", "bf16"):
        for M, N, K in ((1, 1, 4096), (1, 8, 8192), (2, 3, 4096), (1, 16, 4096), (1, 8, 8), (1, 64, 8), (33, 3, 5), (16, 8, 8192)):
            for back in (False, True):
                size = {"M": M, "K": K, "dtype": dtype, "workspace": None, "workspace_bytes": 0}
                for fn, width, ask in (("cgbn_linear", "N", L.cgbn_linear_workspace_bytes), ("cgbn_gated", "F", L.cgbn_gated_workspace_bytes)):
                    nbytes = ask(M, N, K, dtype, back)
                    fn += "_backward" if back else "_forward"
                    if nbytes > 256:
                        assert _code(fn, {**CALLS[fn], **size, width: N, "act": "relu"}) == 6, (fn, M, N, K, dtype)
                        seen += nbytes == 512
                    else:
                        assert not back
        for T, Hq, Hk, D in ((0, 1, 0, 1), (1, 1, 0, 8), (1, 1, 1, 32), (5, 2, 1, 16)):
            nbytes = L.cgbn_head_norm_workspace_bytes(T, Hq, Hk, D, dtype)
            kw = {**CALLS["cgbn_head_norm_backward"], "T": T, "Hq": Hq, "Hk": Hk, "D": D, "R": 0, "dtype": dtype, "workspace": None, "workspace_bytes": 0}
            assert nbytes > 256 and _code("cgbn_head_norm_backward", kw) == 6
    assert seen > 8
    # a call that does without, and one that does not, as they came with 256 bytes each
    assert L.cgbn_linear_workspace_bytes(1, 16, 64, "bf16", False) == 256 and L.cgbn_linear_workspace_bytes(1, 16, 4096, "bf16", False) == 512
    assert L.cgbn_gated_workspace_bytes(1, 8, 8, "bf16", True) > 256


def test_linear_results_over_the_bias_and_the_bias_gradient_over_others():
    _refused("cgbn_linear_forward", [{"bias": 7 * P, "y": 7 * P}, {"bias": 7 * P, "z": 7 * P}], 11)
    _refused("cgbn_linear_backward", [{"dbias": P * at} for at in (1, 2, 3, 4, 5, 6, 8)], 11)
    # no rows: the weights' gradient is zero, and so would the weights be
    _refused("cgbn_linear_backward", [{"M": 0, "dw": 3 * P}, {"M": 0, "dbias": 3 * P}, {"M": 0, "dbias": 6 * P}], 11)
    # what is not wrong is refused for the workspace alone
    for change in ({"dresidual": P}, {"dx": 4 * P}, {"act": 0, "dbias": 4 * P}):
        assert _code("cgbn_linear_backward", {**CALLS["cgbn_linear_backward"], **change, "workspace": None}) == 6, change
    assert _code("cgbn_linear_forward", {**CALLS["cgbn_linear_forward"], "M": 100, "K": 33, "y": 3 * P, "bias": 7 * P, "workspace": None}) == 6
