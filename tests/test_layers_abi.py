"""The layers' entry points without a GPU: sizes, refusals (all before any launch) and the extension's argument marshalling."""

import ctypes

import pytest

from paper_1711_07240_amd import cgbn as L

P = 1 << 20          # an aligned address that is never followed: every call below is refused, or has no rows and nothing to zero

LINEAR_F = dict(x=P, w=2 * P, bias=P, residual=3 * P, M=4, N=16, K=32, act=1, y=4 * P, z=5 * P, dtype=1, workspace=P, workspace_bytes=1 << 30, stream=0)
LINEAR_B = dict(dy=P, x=2 * P, w=3 * P, saved=4 * P, M=4, N=16, K=32, act=1, dx=5 * P, dw=6 * P, dbias=7 * P, dresidual=8 * P, dtype=1, workspace=P,
                workspace_bytes=1 << 30, stream=0)
GATED_F = dict(x=P, w_gate=2 * P, w_up=3 * P, M=4, F=16, K=32, act=3, h=4 * P, gate=5 * P, up=6 * P, dtype=1, workspace=P, workspace_bytes=1 << 30, stream=0)
GATED_B = dict(dh=P, x=2 * P, w_gate=3 * P, w_up=4 * P, gate=5 * P, up=6 * P, M=4, F=16, K=32, act=3, dx=7 * P, dw_gate=8 * P, dw_up=9 * P, dtype=1,
               workspace=P, workspace_bytes=1 << 30, stream=0)
HEAD_F = dict(q=P, ldq=64, k=2 * P, ldk=64, T=4, Hq=2, Hk=1, D=32, R=16, style=0, positions=P, cos=P, sin=P, table_rows=9, wq=P, wk=P, eps=1e-5, yq=3 * P,
              ldyq=64, yk=4 * P, ldyk=32, dtype=1, stream=0)
HEAD_B = dict(dyq=P, lddyq=64, dyk=2 * P, lddyk=32, q=3 * P, ldq=64, k=4 * P, ldk=64, T=4, Hq=2, Hk=1, D=32, R=16, style=0, positions=P, cos=P, sin=P,
              table_rows=9, wq=P, wk=P, eps=1e-5, dq=5 * P, lddq=64, dk=6 * P, lddk=32, dwq=P, dwk=2 * P, dtype=1, workspace=P, workspace_bytes=1 << 30,
              stream=0)
CALLS = {"cgbn_linear_forward": LINEAR_F, "cgbn_linear_backward": LINEAR_B, "cgbn_gated_forward": GATED_F, "cgbn_gated_backward": GATED_B,
         "cgbn_head_norm_forward": HEAD_F, "cgbn_head_norm_backward": HEAD_B}

# what makes a call wrong, and the status that says so
WRONG = {
    "cgbn_linear_forward": [({"x": None}, 1), ({"w": None}, 1), ({"y": None}, 1), ({"M": -1}, 2), ({"M": 1 << 31}, 2), ({"N": 0}, 2), ({"K": -3}, 2),
                            ({"N": 1 << 21}, 2), ({"M": 1 << 30, "N": 1 << 20}, 2), ({"dtype": 2}, 4), ({"act": 4}, 13), ({"act": -1}, 13), ({"x": P + 8}, 7), ({"w": P + 2}, 7), ({"y": P + 4}, 7),
                            ({"residual": P + 8}, 7), ({"z": P + 8}, 7), ({"y": P}, 11), ({"y": 2 * P}, 11), ({"z": 4 * P}, 11), ({"z": P}, 11),
                            ({"M": 100, "K": 33, "workspace": None}, 6), ({"M": 100, "K": 33, "workspace": P + 64}, 6),
                            ({"M": 100, "K": 33, "workspace_bytes": 255}, 6)],
    "cgbn_linear_backward": [({"dy": None}, 1), ({"x": None}, 1), ({"w": None}, 1), ({"saved": None}, 1), ({"N": 0}, 2), ({"dtype": -1}, 4), ({"act": 9}, 13),
                             ({"dx": P + 8}, 7), ({"saved": P + 2}, 7), ({"dresidual": P + 2}, 7), ({"dx": P}, 11), ({"dx": 2 * P}, 11), ({"dw": 5 * P}, 11),
                             ({"dw": 3 * P}, 11), ({"dresidual": 2 * P}, 11), ({"dresidual": 5 * P}, 11), ({"workspace": None}, 6),
                             ({"workspace_bytes": 0}, 6)],
    "cgbn_gated_forward": [({"x": None}, 1), ({"w_gate": None}, 1), ({"w_up": None}, 1), ({"h": None}, 1), ({"gate": None}, 1), ({"up": None}, 1), ({"F": 0}, 2),
                           ({"M": -5}, 2), ({"dtype": 7}, 4), ({"act": 5}, 13), ({"h": P + 8}, 7), ({"h": 5 * P}, 11), ({"gate": 6 * P}, 11), ({"h": P}, 11),
                           ({"up": 2 * P}, 11), ({"M": 64, "K": 31, "workspace_bytes": 16}, 6)],
    "cgbn_gated_backward": [({"dh": None}, 1), ({"gate": None}, 1), ({"up": None}, 1), ({"dw_gate": None}, 1), ({"K": 0}, 2), ({"dtype": 3}, 4), ({"act": 4}, 13),
                            ({"dx": P + 2}, 7), ({"dw_up": 8 * P}, 11), ({"dx": 2 * P}, 11), ({"dw_gate": 5 * P}, 11), ({"workspace": None}, 6),
                            ({"workspace_bytes": 64}, 6)],
    "cgbn_head_norm_forward": [({"q": None}, 1), ({"k": None}, 1), ({"wq": None}, 1), ({"wk": None}, 1), ({"yq": None}, 1), ({"cos": None}, 1), ({"sin": None}, 1),
                               ({"T": -1}, 2), ({"Hq": 0}, 2), ({"Hk": -1}, 2), ({"D": 0}, 2), ({"D": 1025}, 2), ({"R": 15}, 2), ({"R": 34}, 2), ({"R": -2}, 2),
                               ({"table_rows": 0}, 2), ({"dtype": 2}, 4), ({"eps": 0.0}, 5), ({"eps": float("nan")}, 5), ({"eps": float("inf")}, 5), ({"style": 2}, 13),
                               ({"ldq": 63}, 14), ({"ldyk": 31}, 14), ({"ldk": -64}, 14), ({"q": P + 1}, 7), ({"yq": P, "ldyq": 80}, 11), ({"yk": 3 * P}, 11)],
    "cgbn_head_norm_backward": [({"dyq": None}, 1), ({"dk": None}, 1), ({"dwq": None}, 1), ({"dwk": None}, 1), ({"D": 2000}, 2), ({"lddq": 10}, 14),
                                ({"lddyk": 31}, 14), ({"dwk": P}, 11), ({"dq": P, "lddq": 70}, 11), ({"dk": 5 * P}, 11), ({"eps": -1.0}, 5),
                                ({"workspace": None}, 6), ({"workspace": P + 128}, 6), ({"workspace_bytes": 100}, 6)],
}


def _code(fn, kw):
    try:
        getattr(L, fn)(**kw)
    except L.CgbnError as e:
        return e.code
    return L.CGBN_OK


@pytest.mark.parametrize("fn", CALLS)
def test_refusals_by_the_extension_and_by_ctypes(fn):
    for change, want in WRONG[fn]:
        kw = {**CALLS[fn], **change}
        assert _code(fn, kw) == want, (fn, change)
        assert getattr(L.lib(), fn)(*kw.values()) == want, (fn, change)


class Buffer:
    """What the binding asks of a tensor."""
    def __init__(self, address, count=0, size=1):
        self.address, self.count, self.size = address, count, size

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.count

    def element_size(self):
        return self.size


def test_names_tensors_and_sizes():
    kw = {**LINEAR_B, "act": "gelu", "dtype": "bf16", "x": Buffer(2 * P), "workspace": Buffer(P, 3, 4), "workspace_bytes": None}
    assert _code("cgbn_linear_backward", kw) == 6
    assert _code("cgbn_head_norm_forward", {**HEAD_F, "style": "interleaved", "dtype": "f32", "q": Buffer(P + 2)}) == 7
    # (a number of another type goes through ctypes and is refused or taken there)
    assert _code("cgbn_linear_forward", {**LINEAR_F, "M": ctypes.c_longlong(-1)}) == 2
    for bad, error in (({"act": "tanh"}, KeyError), ({"x": "text"}, AttributeError), ({"N": 2.5}, ctypes.ArgumentError)):
        with pytest.raises(error):
            L.cgbn_linear_forward(**{**LINEAR_F, **bad})


def test_without_rows_nothing_is_asked_for():
    for fn in ("cgbn_linear_forward", "cgbn_gated_forward"):
        kw = {k: (None if v is not None and k in ("x", "y", "z", "h", "gate", "up", "residual", "workspace") else v) for k, v in CALLS[fn].items()}
        assert _code(fn, {**kw, "M": 0, "workspace_bytes": 0}) == L.CGBN_OK
    kw = {k: (None if k in ("q", "k", "yq", "yk") else v) for k, v in HEAD_F.items()}
    assert _code("cgbn_head_norm_forward", {**kw, "T": 0}) == L.CGBN_OK


def test_workspace_sizes():
    for fn in (L.cgbn_linear_workspace_bytes, L.cgbn_gated_workspace_bytes):
        for dtype in ("f32", "bf16"):
            for size in ((0, 8, 8), (1, 4096, 4096), (300, 17, 33), (5000, 4096, 1000), (268800, 128, 512)):
                f, b = fn(*size, dtype, False), fn(*size, dtype, True)
                assert f >= 256 and f % 256 == 0 and b >= 256 and b % 256 == 0
                assert b < 8 * sum((size[0] * size[1] * 2, size[0] * size[2], size[1] * size[2] * 2)) + (1 << 30)
        assert fn(-1, 8, 8, "f32", False) == 0 and fn(8, 0, 8, "f32", True) == 0 and fn(8, 8, 8, 7, False) == 0 and fn(1 << 30, 1 << 20, 8, 0, False) == 0
    # rows of whole chunks and enough tiles: nothing is copied, nothing is split
    assert L.cgbn_linear_workspace_bytes(65536, 4096, 4096, "bf16", False) == 256
    assert L.cgbn_head_norm_workspace_bytes(5, 2, 1, 64, "bf16") > 0 and L.cgbn_head_norm_workspace_bytes(5, 0, 1, 64, "bf16") == 0


def test_statuses_of_the_layers():
    assert {L.cgbn_status_string(13), L.cgbn_status_string(14)}.isdisjoint({"unknown status"})
    assert L.cgbn_status_string(15) == "unknown status"
