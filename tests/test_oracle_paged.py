"""The paged cache's and beam search's references on cases worked out by hand."""

import math

import numpy as np

from oracle.paged import assign_pages, beam_values, best, take_over


def test_pages_go_back_first_and_come_off_the_top():
    table = [[5, 6, -1], [7, 8, 9], [-1, -1, -1]]
    # Sequence 1 shrank to one page, 0 stays, 2 starts with three rows.
    got = assign_pages(2, 10, table, [2, 3, 0], [0, 1] + [-9] * 8, 2, [3, 1, 0], [1, 1, 3], 3, 6)
    assert got == ([[5, 6, -1], [7, 8, 9], [9, 8, -1]], [2, 1, 2], [0, 1, 8, 9] + [-9] * 6, 2,
                   [[13, -1, -1], [15, -1, -1], [18, 19, 16]], 0)


def test_those_who_get_none_keep_what_they_hold():
    table = [[-1, -1], [4, -1], [-1, -1]]
    got = assign_pages(1, 5, table, [0, 1, 0], [0, 1, 2, 3, -9], 1, [0, 1, 0], [2, 0, 1], 2, 2)
    assert got == (table, [0, 1, 0], [0, 1, 2, 3, -9], 1, [[-1, -1], [-1, -1], [-1, -1]], 2)


def test_shared_pages_do_not_go_back():
    got = assign_pages(4, 6, [[1, 2, 3]], [3], [0, 5, -9, -9, -9, -9], 2, [0], [0], 1, 12, shared=[2])
    assert got == ([[1, 2, 3]], [0], [0, 5, 3, -9, -9, -9], 3, [[-1]], 0)


def test_rows_past_L_have_no_slot():
    table, held, _, n, slots, _ = assign_pages(4, 8, [[0, 1, -1]], [2], [6, 7], 2, [-1], [9], 9, 6)
    assert (held, n, slots) == ([2], 2, [[-1, 0, 1, 2, 3, 4, 5, -1, -1]])


def test_beam_values():
    x = np.log([1.0, 2.0, 1.0])
    v, err = beam_values(x, -1.0)
    assert np.allclose(v, -1.0 + np.log([0.25, 0.5, 0.25])) and 0 < err < 1e-5
    assert beam_values(x, -1.0, True, 2)[0].tolist() == [-math.inf, -math.inf, -1.0]
    assert (beam_values(x, -math.inf)[0] == -math.inf).all()
    assert beam_values([math.inf, math.nan, math.inf, 0], 0.0)[0].tolist() == [-math.log(2), -math.inf, -math.log(2), -math.inf]
    assert best([[1.0, 2.0], [2.0, -math.inf]], 4) == ([0, 1, 0, -1], [1, 0, 0, -1], [2.0, 2.0, 1.0, -math.inf])


def test_take_over():
    # Beam 1 goes on three times, 3 once; 0 and 2 end.
    assert take_over([1, 1, 3, 1], [5, 6, 7, 8], None, 4, 4, 16) == [(1, 6, 0), (0, 6, 6), (3, 8, 0), (2, 6, 6)]
    assert take_over([-1, 0, 9], [5, 6, 7], [1, 2, 2], 2, 4, 16) == [(1, 0, 0), (0, 4, 0), (2, 0, 0)]
    # A copy ends where the parent's pages or the child's do.
    assert take_over([0, 0, 2, 2], [9, 9, 9, 9], [2, 1, 1, 3], 3, 4, 16) == [(0, 8, 0), (1, 4, 4), (2, 4, 0), (3, 4, 4)]
