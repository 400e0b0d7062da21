"""Block tables of beams that are refused, where the beams of a request hold different numbers of pages: rows come out as
they were, and what lies behind them untouched."""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_beams import beam_state, both

pytestmark = pytest.mark.gpu


def test_a_short_row_that_would_have_taken_over_a_long_one():
    for table, lengths, page, kept in (([[10, 11, 12], [20, -1, -1]], [40, 5], 16, 1), ([[10, 11, 12], [13, -1, -1]], [20, 3], 8, 3),
                                       ([[10, 11, 12], [-1, -1, -1]], [33, 0], 16, 0)):
        # with a page it is served, without one its row is as it was
        for free in ([], [7]):
            got, want = both(np.array([0, 0]), np.array(lengths), np.array(table), 2, page, np.array(free, dtype=int), len(free), 4, 64,
                             np.array([kept]))
            held = -(-lengths[1] // page)
            released = held > kept
            assert want["short"] == (not free and not released)
            if want["short"]:
                assert got["table"][1].tolist() == table[1][:held] + [-7] * (3 - held) and not got["lengths"].any()


@pytest.mark.parametrize("beams,n,page,longest", [(4, 9, 16, 70), (3, 1200, 16, 70), (8, 5, 8, 5000), (9, 6, 8, 4200), (32, 7, 16, 300),
                                                  (2, 3, 256, 1000), (1, 5, 16, 90)])
@pytest.mark.parametrize("count", [0, 1, 2, 5, 13])
def test_requests_that_are_refused_and_served_side_by_side(beams, n, page, longest, count):
    rng = np.random.default_rng(100 * count + beams)
    refused = 0
    for kind in range(3):
        lengths, table, free, total = beam_state(rng, n, beams, page, longest)
        if kind == 2:  # a search begins: one beam is there, and all come from it
            lengths = np.where(np.arange(n * beams) % beams, 0, lengths)
            parents = np.zeros(n * beams, dtype=int)
        else:
            parents = np.maximum((rng.random(n * beams) ** 3 * (beams + 1)).astype(int) - kind, -kind)
            parents = np.minimum(parents, beams - 1)
        kept = rng.integers(0, 400, n) if kind == 1 else None
        _, want = both(parents, lengths, table, beams, page, free, min(count, len(free)), total, total, kept)
        refused += want["short"]
    assert refused or beams == 1 or count > n * (beams - 1) or count >= 5


def test_as_many_pages_as_the_rows_can_need_and_one_less():
    rng = np.random.default_rng(8)
    n, beams = 6, 5
    for most in (n * (beams - 1), n * (beams - 1) - 1):
        lengths = np.where(np.arange(n * beams) % beams, 0, 21)
        table = np.full((n * beams, 3), -1)
        table[::beams, :2] = 100 + np.arange(2 * n).reshape(n, 2)
        _, want = both(np.zeros(n * beams, dtype=int), lengths, table, beams, 16, rng.permutation(90)[:most], most, 120, 200)
        assert want["short"] == (most < n * (beams - 1)) and want["left"] in (0, beams - 2)
