"""The serving operators' entry points without a GPU: sizes, refusals (all before any launch), the binding, the frequencies, and closed values of
their oracle."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import serving_oracle as V
from paper_1711_07240_amd import cgbn as L

# (a call that is wrongly taken would follow addresses that are none)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU")
P = 1 << 20          # an aligned address that is never followed: every call below is refused, or has nothing to do

ROTATE = dict(q=P, ldq=64, k=2 * P, ldk=64, T=4, Hq=2, Hk=1, D=32, R=16, style=0, positions=5 * P, freq=6 * P, magnitude=1.0, yq=3 * P, ldyq=64, yk=4 * P,
              ldyk=32, dtype=1, stream=0)
BACK = {{"q": "dyq", "ldq": "lddyq", "k": "dyk", "ldk": "lddyk", "yq": "dq", "ldyq": "lddq", "yk": "dk", "ldyk": "lddk"}.get(k, k): v
        for k, v in ROTATE.items()}
PLAN = dict(have=P, fresh=2 * P, B=5000, before=0, free_pages=3 * P, free_count=9, taken=4 * P, counts=5 * P, table=6 * P, max_pages=4, pages=9, page=16, T=70,
            rows=7 * P, lengths=8 * P, slots=9 * P, positions=10 * P, workspace=P, workspace_bytes=1 << 30, stream=0)
STORE = dict(k=P, ldk=256, v=2 * P, ldv=256, T=4, Hk=2, D=64, slots=3 * P, k_pages=4 * P, v_pages=5 * P, pages=9, page=16, dtype=1, stream=0)
ATTEND = dict(q=P, ldq=256, T=4, B=4, rows=None, lengths=2 * P, Hq=4, Hk=2, D=64, scale=0.125, k_pages=3 * P, v_pages=4 * P, pages=9, page=16,
              prefix_table=5 * P, prefix=700, table=6 * P, max_pages=40, out=7 * P, ldo=256, lse=8 * P, dtype=1, workspace=9 * P, workspace_bytes=1 << 30, stream=0)
CALLS = {"cgbn_rotate_forward": ROTATE, "cgbn_rotate_backward": BACK, "cgbn_page_plan": PLAN, "cgbn_page_store": STORE, "cgbn_prefix_attention": ATTEND}

# what makes a call wrong, and the status that says so
WRONG = {
    "cgbn_rotate_forward": [({"q": None}, 1), ({"k": None}, 1), ({"yq": None}, 1), ({"yk": None}, 1), ({"freq": None}, 1), ({"T": -1}, 2), ({"Hq": 0}, 2),
                            ({"Hk": -1}, 2), ({"D": 0}, 2), ({"D": 1025}, 2), ({"R": 15}, 2), ({"R": 34}, 2), ({"R": -2}, 2), ({"dtype": 2}, 4), ({"style": 2}, 13),
                            ({"ldq": 63}, 14), ({"ldyk": 31}, 14), ({"ldk": -64}, 14), ({"q": P + 1}, 7), ({"freq": 6 * P + 4}, 7), ({"positions": 5 * P + 2}, 7),
                            ({"yq": P, "ldyq": 80}, 11), ({"yk": 3 * P}, 11), ({"yq": 2 * P}, 11), ({"yk": P}, 11), ({"yq": 5 * P}, 11), ({"yk": 6 * P}, 11),
                            ({"T": 1 << 30, "Hq": 9}, 2)],
    "cgbn_rotate_backward": [({"dyq": None}, 1), ({"dk": None}, 1), ({"lddyk": 31}, 14), ({"dq": 2 * P}, 11), ({"style": -1}, 13), ({"R": 33}, 2)],
    "cgbn_page_plan": [({"have": None}, 1), ({"fresh": None}, 1), ({"free_pages": None}, 1), ({"taken": None}, 1), ({"counts": None}, 1), ({"table": None}, 1),
                       ({"rows": None}, 1), ({"lengths": None}, 1), ({"slots": None}, 1), ({"positions": None}, 1), ({"B": -1}, 2), ({"B": (1 << 20) + 1}, 2),
                       ({"before": -1}, 2), ({"before": (1 << 30) + 1}, 2), ({"max_pages": 0}, 2), ({"max_pages": 65537}, 2), ({"page": 0}, 2), ({"page": 24}, 2),
                       ({"page": 2048}, 2), ({"pages": -1}, 2), ({"pages": 1 << 27}, 2), ({"free_count": -1}, 2), ({"free_count": 1 << 30}, 2), ({"T": -1}, 2),
                       ({"T": (1 << 29) + 1}, 2), ({"have": P + 2}, 7), ({"positions": P + 1}, 7), ({"slots": 10 * P}, 11), ({"rows": P}, 11),
                       ({"lengths": 7 * P}, 11), ({"table": 3 * P}, 11), ({"counts": 2 * P}, 11), ({"slots": 4 * P}, 11), ({"workspace": None}, 6),
                       ({"workspace": P + 64}, 6), ({"workspace_bytes": 19999}, 6)],
    "cgbn_page_store": [({"k": None}, 1), ({"v": None}, 1), ({"slots": None}, 1), ({"k_pages": None}, 1), ({"v_pages": None}, 1), ({"T": -1}, 2), ({"Hk": 0}, 2),
                        ({"Hk": 1025}, 2), ({"D": 4}, 2), ({"D": 60}, 2), ({"D": 264}, 2), ({"page": 3}, 2), ({"pages": 1 << 28}, 2), ({"dtype": 2}, 4), ({"ldk": 127}, 14),
                        ({"ldv": -256}, 14), ({"k": P + 8}, 7), ({"v_pages": 5 * P + 4}, 7), ({"ldk": 260}, 7), ({"slots": 3 * P + 1}, 7), ({"v_pages": 4 * P}, 11),
                        ({"k_pages": P}, 11), ({"v_pages": P}, 11), ({"k_pages": 3 * P}, 11)],
    "cgbn_prefix_attention": [({"q": None}, 1), ({"out": None}, 1), ({"k_pages": None}, 1), ({"v_pages": None}, 1), ({"prefix_table": None}, 1), ({"table": None}, 1),
                              ({"lengths": None}, 1), ({"T": -1}, 2), ({"T": 5}, 2), ({"B": -1}, 2), ({"Hq": 5}, 2), ({"Hq": 0}, 2), ({"Hk": 0}, 2), ({"Hq": 1026}, 2),
                              ({"D": 4}, 2), ({"D": 65}, 2), ({"D": 264}, 2), ({"page": 12}, 2), ({"page": 2048}, 2), ({"pages": -1}, 2), ({"pages": 1 << 27}, 2),
                              ({"prefix": -1}, 2), ({"max_pages": -1}, 2), ({"max_pages": 1 << 27}, 2), ({"T": 1 << 25, "rows": 11 * P}, 2), ({"dtype": 2}, 4),
                              ({"ldq": 255}, 14), ({"ldo": 0}, 14), ({"q": P + 8}, 7), ({"out": 7 * P + 2}, 7), ({"ldq": 260}, 7), ({"lse": 8 * P + 2}, 7),
                              ({"rows": P + 2}, 7), ({"out": P}, 11), ({"out": 3 * P}, 11), ({"lse": 7 * P}, 11), ({"lse": 2 * P}, 11), ({"out": 9 * P}, 11),
                              ({"workspace": None}, 6), ({"workspace": P + 64}, 6), ({"workspace_bytes": 100}, 6)],
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


def test_names_tensors_and_sizes():
    class Buffer:
        def __init__(self, address, count=0, size=1):
            self.address, self.count, self.size = address, count, size

        def data_ptr(self):
            return self.address

        def numel(self):
            return self.count

        def element_size(self):
            return self.size

    assert _code("cgbn_prefix_attention", {**ATTEND, "dtype": "bf16", "q": Buffer(P), "workspace": Buffer(9 * P, 3, 4), "workspace_bytes": None}) == 6
    assert _code("cgbn_page_plan", {**PLAN, "workspace": Buffer(P, 3, 4), "workspace_bytes": None}) == 6
    assert _code("cgbn_rotate_forward", {**ROTATE, "style": "interleaved", "dtype": "f32", "q": Buffer(P + 2)}) == 7
    # (a number of another type goes through ctypes and is refused or taken there)
    assert _code("cgbn_page_store", {**STORE, "T": ctypes.c_longlong(-1)}) == 2
    assert _code("cgbn_prefix_attention", {**ATTEND, "scale": 1, "T": -1}) == 2
    for bad, error in (({"style": "sideways"}, KeyError), ({"q": "text"}, AttributeError), ({"Hq": 2.5}, ctypes.ArgumentError)):
        with pytest.raises(error):
            L.cgbn_rotate_forward(**{**ROTATE, **bad})


def test_without_rows_nothing_is_asked_for():
    assert _code("cgbn_rotate_forward", {**ROTATE, "T": 0, "q": None, "yq": None, "freq": None}) == 0
    assert _code("cgbn_page_store", {**STORE, "T": 0, "k": None, "slots": None}) == 0
    for change in ({"T": 0, "B": 0}, {"T": 0, "rows": P}, {"B": 0, "rows": P}):
        assert _code("cgbn_prefix_attention", {**ATTEND, "q": None, "out": None, "workspace": None, **change}) == 0
    # nothing to turn, in place: nothing to do
    assert _code("cgbn_rotate_forward", {**ROTATE, "R": 0, "yq": P, "yk": 2 * P, "ldyk": 64, "freq": None}) == 0


def test_workspace_sizes():
    for dtype in ("f32", "bf16"):
        for size in ((1, 1, 8, 8, 64, 100, 64), (64, 64, 32, 8, 128, 32768, 2048), (4, 4, 32, 8, 128, 0, 1 << 20), (5000, 16, 32, 8, 128, 8192, 1024), (7, 3, 4, 4, 8, 0, 16)):
            n = L.cgbn_prefix_attention_workspace_bytes(*size, dtype)
            assert n >= 256 and n % 256 == 0 and n <= 128 * (size[0] * size[2] * (size[4] + 2) * 4) + 256
    assert L.cgbn_prefix_attention_workspace_bytes(0, 0, 8, 8, 64, 0, 0, "f32") == 256
    for bad in ((-1, 1, 8, 8, 64, 0, 0), (1, 1, 9, 8, 64, 0, 0), (1, 1, 8, 8, 63, 0, 0), (1, 1, 8, 8, 64, -1, 0), (1 << 24, 1, 8, 8, 64, 0, 0)):
        assert L.cgbn_prefix_attention_workspace_bytes(*bad, "bf16") == 0
    assert L.cgbn_prefix_attention_workspace_bytes(1, 1, 8, 8, 64, 0, 0, 7) == 0
    assert L.cgbn_page_plan_workspace_bytes(16, 16) == 256 and L.cgbn_page_plan_workspace_bytes(5000, 16) == 20224
    assert L.cgbn_page_plan_workspace_bytes(1, 1 << 20) == 512 and L.cgbn_page_plan_workspace_bytes(-1, 0) == 0
    # many requests in tables for far more keys than most have: by the workgroups, not by the parts that each may have
    for B, Hq, Hk in ((256, 64, 8), (1024, 64, 2), (64, 32, 8)):
        assert L.cgbn_prefix_attention_workspace_bytes(B, B, Hq, Hk, 128, 0, 65536, "bf16") < 100 << 20
    # of one request after the other, with the workspace asked for: refused for something that is looked at later, never for it
    for T, B, rows in ((64, 64, None), (64, 64, 11 * P), (70, 9, 11 * P), (5000, 3, 11 * P)):
        n = L.cgbn_prefix_attention_workspace_bytes(T, B, 4, 2, 64, 700, 640, 1)
        kw = {**ATTEND, "T": T, "B": B, "rows": rows, "workspace_bytes": n}
        assert _code("cgbn_prefix_attention", {**kw, "workspace": None}) == (6 if n > 256 else 8)


# ---- frequencies ----


def _frequencies(R, base, *rest):
    f = np.full(R // 2 + 1, 7.0)
    L.cgbn_rotary_frequencies(R, base, *rest, f.ctypes.data)
    assert f[-1] == 7.0
    return f[:-1]


@pytest.mark.parametrize("R", [0, 2, 4, 32, 128, 1024])
def test_frequencies(R):
    for scaling in ("none", "positions", "base", "parts"):
        for factor, base in ((1.0, 10000.0), (8.0, 500000.0), (40.0, 3.0)):
            got = _frequencies(R, base, scaling, factor, 4096.0, 32.0, 1.0)
            want = V.frequencies(R, base, scaling, factor, 4096.0, 32.0, 1.0)
            # a power is off by a few units of its logarithm, up to 20 here
            assert np.all(np.abs(got - want) <= 40 * 2.0 ** -52 * want)
            if factor == 1.0:
                assert np.all(np.abs(got - V.frequencies(R, base)) <= 40 * 2.0 ** -52 * want)


def test_frequencies_by_their_meaning():
    """The slowest pair: positions and by parts divide it by the factor, a larger base too; the fastest is left alone but by positions."""
    plain = _frequencies(128, 10000.0, "none", 1.0, 0.0, 0.0, 0.0)
    assert plain[0] == 1.0 and abs(plain[32] - 0.01) < 1e-16
    for scaling, first in (("positions", 0.125), ("base", 1.0), ("parts", 1.0)):
        f = _frequencies(128, 10000.0, scaling, 8.0, 4096.0, 32.0, 1.0)
        assert abs(f[-1] / plain[-1] * 8.0 - 1) < 1e-13 and f[0] == first
    half = _frequencies(4, (4096 / (2 * math.pi) / 16.5) ** 2, "parts", 3.0, 4096.0, 32.0, 1.0)        # a pair of 16.5 turns, between 1 and 32
    assert abs(half[1] * 4096 / (2 * math.pi) - 16.5 * (0.5 + 0.5 / 3)) < 1e-12


def test_frequencies_refused():
    f = np.zeros(8).ctypes.data
    good = (16, 10000.0, 3, 8.0, 4096.0, 32.0, 1.0, f)
    assert L.lib().cgbn_rotary_frequencies(*good) == 0
    for at, value, code in ((0, -2, 2), (0, 15, 2), (0, 1026, 2), (1, 1.0, 2), (1, math.inf, 2), (1, math.nan, 2), (2, 4, 13), (2, -1, 13), (3, 0.5, 2), (3, math.nan, 2),
                            (3, math.inf, 2), (4, 0.0, 2), (5, 1.0, 2), (5, math.inf, 2), (6, -1.0, 2), (6, math.nan, 2), (7, None, 1)):
        bad = list(good)
        bad[at] = value
        assert L.lib().cgbn_rotary_frequencies(*bad) == code, (at, value)
    L.cgbn_rotary_frequencies(16, 10000, "none", math.nan, math.nan, math.nan, math.nan, torch.empty(8, dtype=torch.float64))      # looked at by none


# ---- the oracle's own values ----


def test_oracle_rotation():
    x = np.array([[1.0, 2.0, 3.0, 4.0, 5.0]])
    quarter = [math.pi / 2, math.pi]
    np.testing.assert_allclose(V.rotate(x, 1, 5, 4, "halves", [1], quarter, 2.0), [[-6.0, -4.0, 2.0, -8.0, 5.0]], atol=1e-14)
    np.testing.assert_allclose(V.rotate(x, 1, 5, 4, "interleaved", [1], quarter, 2.0), [[-4.0, 2.0, -6.0, -8.0, 5.0]], atol=1e-14)
    turned = V.rotate(x, 1, 5, 4, "halves", [3], [0.3, 0.7], 1.0)
    np.testing.assert_allclose(V.rotate(turned, 1, 5, 4, "halves", [3], [0.3, 0.7], 1.0, back=True), x, atol=1e-14)


def test_oracle_plan():
    rows, lengths, table, slots, positions, counts = V.plan([3, 0, 4], [2, 0, 1], 10, [7, 5, 6], 1, [[2, -1], [-1, -1], [4, -1]], 2, 8, 4, 5)
    assert rows == [0, 2, 2, 3] and lengths == [5, 0, 5]
    assert table.tolist() == [[2, 5], [-1, -1], [4, 6]]
    assert slots == [11, 20, 24, -1, -1] and positions == [13, 14, 14, 0, 0] and counts == [3, 0]
    # the list ends: a page's later tokens have no place either; the table ends; the rows end
    assert V.plan([0, 0], [2, 1], 0, [3], 0, [[-1], [-1]], 1, 8, 4, 9)[3:] == ([12, 13] + [-1] * 7, [0, 1, 0] + [0] * 6, [1, 1])
    assert V.plan([4], [2], 0, [3], 0, [[1]], 1, 8, 4, 9)[5] == [0, 2]
    assert V.plan([0], [7], 0, [3, 2], 0, [[-1] * 4], 4, 8, 4, 5)[0::5] == ([0, 5], [2, 2])


def test_oracle_store_and_attention():
    pool = V.store(np.arange(8.0).reshape(2, 4), 2, 2, [5, -1], np.zeros((2, 2, 4, 2)))
    assert pool[1, 0, 1].tolist() == [0.0, 1.0] and pool[1, 1, 1].tolist() == [2.0, 3.0] and pool.sum() == 6.0
    o, lse, w = V.attention(np.array([2.0, 0.0]), np.array([[math.log(3.0), 9.0], [0.0, 1.0]]), np.array([[4.0, 8.0], [0.0, 4.0]]), 0.5)
    np.testing.assert_allclose(o, [3.0, 7.0])
    assert abs(lse - math.log(4.0)) < 1e-15 and abs(w[0] - 0.75) < 1e-15
    o, lse, _ = V.attention(np.ones(2), np.zeros((0, 2)), np.zeros((0, 2)), 1.0)
    assert o.tolist() == [0.0, 0.0] and lse == -math.inf
