"""The block's cache in pages without a GPU: the library's calls are written down instead of made."""

import pytest
import torch

from paper_1711_07240_amd import block as B
from paper_1711_07240_amd import cgbn as L

LAUNCH = ["frozen_forward", "linear_forward", "gated_forward", "head_norm_forward", "rotate_forward", "page_plan", "page_store", "prefix_attention"]


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in LAUNCH:
        monkeypatch.setattr(L, "cgbn_" + name, lambda *args, _name=name: made.append((_name, args)))
    return made


def _pages(dtype="f32", rows=6, pages=30):
    blk = B.Block(channels=64, heads=2, head_size=32, width=96, positions=128, dtype=dtype, device="cpu")
    return blk, B.Pages(blk, requests=3, rows=rows, pages=pages, page=4, most=6)


def _rows(n, blk, channels=64):
    return torch.ones(n, channels, dtype=blk.dt)


def test_rows_of_another_size_or_type_are_refused(calls):
    """More rows than the plan has slots for would be stored by what lies behind them; values of half the size would be read past their end."""
    blk, pages = _pages()
    for x in (_rows(7, blk), _rows(0, blk), _rows(6, blk, 63), _rows(6, blk).bfloat16(), _rows(12, blk)[::2], _rows(6, blk).flatten()):
        with pytest.raises(ValueError):
            pages.step(x)
    for x in (_rows(9, blk, 65), _rows(9, blk).bfloat16(), _rows(18, blk)[::2], _rows(9, blk).flatten()):
        with pytest.raises(ValueError):
            pages.share(x)
    assert not calls
    pages.share(_rows(9, blk))
    pages.step(_rows(6, blk))
    assert [name for name, _ in calls].count("prefix_attention") == 2


def test_the_prefix_is_shared_once_and_first(calls):
    """A second one would take the first one's place, with positions behind it; after a step requests' tokens stand where it belongs."""
    blk, pages = _pages()
    with pytest.raises(ValueError):
        pages.share(_rows(121, blk))                    # one token more than there are pages for
    assert pages.share(_rows(0, blk)).shape == (0, 64) and not calls and pages.prefix == 0
    pages.share(_rows(120, blk))
    with pytest.raises(ValueError):
        pages.share(_rows(4, blk))
    assert pages.prefix == 120 and pages.prefix_table.numel() == 30
    blk, pages = _pages()
    pages.step(_rows(6, blk))
    made = len(calls)
    with pytest.raises(ValueError):
        pages.share(_rows(4, blk))
    assert len(calls) == made


def _workspaces(made):
    at = {"linear_forward": 11, "gated_forward": 11}
    return [(name, args[at[name]].data_ptr(), args[at[name]].numel()) for name, args in made if name in at]


def test_a_step_keeps_its_workspaces(calls):
    """A captured step goes on using them, so what the block does beside it must not take them or put others in their place."""
    blk, pages = _pages("bf16", rows=300, pages=90)
    pages.share(_rows(33, blk))
    del calls[:]
    pages.step(_rows(300, blk))
    first = _workspaces(calls)
    del calls[:]
    blk._linear(_rows(40000, blk), blk.p["o"])
    blk._linear(_rows(1, blk), blk.p["o"])
    blk._gated(_rows(300, blk), False)
    theirs = {at for _, at, _ in _workspaces(calls)}
    del calls[:]
    pages.step(_rows(300, blk))
    assert _workspaces(calls) == first and len(first) == 4
    assert not theirs & {at for _, at, _ in first}
    other = B.Pages(blk, requests=3, rows=300, pages=90, page=4, most=6)
    del calls[:]
    other.step(_rows(300, blk))
    assert not {at for _, at, _ in _workspaces(calls)} & {at for _, at, _ in first}


def test_a_step_of_fewer_rows(calls):
    """The plan cuts tokens at the rows that there are; a captured step's workspaces stay when one of more rows needs larger ones."""
    blk, pages = _pages("bf16", rows=300, pages=90)
    pages.step(_rows(2, blk))
    first, room = _workspaces(calls), pages.room.data_ptr()
    plan, store, attend = (next(args for name, args in calls if name == n) for n in ("page_plan", "page_store", "prefix_attention"))
    assert plan[12] == 2 and plan[15].numel() == plan[16].numel() == 2 and store[4] == 2 and store[7].numel() == 2 and attend[2] == 2
    assert pages.step(_rows(300, blk)).shape == (300, 64)
    kept = {t.data_ptr() for t in (pages.room, pages.layers, *pages.kept)}
    assert {at for _, at, _ in first} | {room} <= kept
