"""oracle/beams.py: what is reported although nothing is offered, and a stack whose count cannot be."""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import beams as ob


@pytest.mark.parametrize("score,done", [(-math.inf, False), (-math.inf, True), (-1.0, True), (-1.0, False)])
@pytest.mark.parametrize("weight,fault", [(1.0, False), (0.0, True), (-2.0, True), (math.inf, True), (math.nan, True)])
def test_a_weight_is_looked_at_in_every_row(score, done, weight, fault):
    tokens, *_, bad = ob.select([[0, 1]], [score], 2, 1, end=1, done=[done], weights=[weight])
    assert bad == fault
    assert (tokens == -1).all() == (fault or score == -math.inf)


@pytest.mark.parametrize("count", [-1, 5])
def test_a_count_that_cannot_be_refuses_every_request(count):
    table, free = [[1, 2], [3, -1]], [9, 8, 7, 6]
    got = ob.pages([0, 0], [6, 3], table, 2, 4, free, count, 4, 20)
    assert got["table"].tolist() == [[1, 2], [3, -7]] and got["free"].tolist() == free and got["left"] == 0
    assert got["bad"] and not got["short"] and not got["lengths"].any() and not np.any(got["copies"])
    assert not ob.pages([0, 0], [6, 3], table, 2, 4, free, 4, 4, 20)["bad"]
