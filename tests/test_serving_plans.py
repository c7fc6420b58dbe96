"""Closed values of the plan's oracle where tokens get no place: counts[1] has every one of them, in the step in which the pages end and in those after it."""

from oracle import serving_oracle as V


def test_steps_after_the_list_has_ended():
    have, table, taken = [8], [[0, 1, -1, -1]], 2
    for step in range(4):
        rows, have, table, slots, _, (taken, without) = V.plan(have, [1], 0, [0, 1], taken, table, 4, 9, 4, 1)
        assert slots == [-1] and without == 1 and taken == 2 and have == [9 + step]
        assert table.tolist() == [[0, 1, -1, -1]]


def test_pages_that_are_not_there():
    # of the list: the second new page is none; of the table: the page that takes the first new tokens is none
    assert V.plan([0], [7], 0, [3, 9, 1], 0, [[-1] * 4], 4, 9, 2, 9)[3::2] == ([6, 7, -1, -1, 2, 3, -1, -1, -1], [3, 3])
    assert V.plan([3], [3], 0, [5], 0, [[0, -7]], 2, 9, 2, 3)[3::2] == ([-1, -1, -1], [0, 3])
    assert V.plan([3], [3], 0, [5], 0, [[0, 9, -1]], 3, 9, 2, 4)[3::2] == ([-1, 10, 11, -1], [1, 1])


def test_every_token_is_counted_once():
    """Rows that end, a table that ends, a list that ends, each cutting off some."""
    rows, lengths, table, slots, _, counts = V.plan([1, 4, 0], [3, 3, 9], 0, [7, 6], 0, [[2, -1], [0, 1], [-1, -1]], 2, 9, 2, 10)
    assert rows == [0, 3, 6, 10] and lengths == [4, 7, 4]
    assert slots == [5, 14, 15, -1, -1, -1, 12, 13, -1, -1] and counts == [2, 3 + 2 + 5]
