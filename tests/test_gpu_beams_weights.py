"""Beam selection reports a weight that is not positive and finite whatever its row offers."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import beams as ob
from test_gpu_beams import DTYPES, INF, check_select, made, run_select

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_a_weight_that_is_none_is_reported_whatever_its_row_offers(dtype):
    rng = np.random.default_rng(6)
    x, _ = made(rng, 6, 900, dtype)
    for weight in (0.0, -1.0, INF, float("nan")):
        for score, ended in ((-INF, False), (-INF, True), (-1.0, True), (-1.0, False)):
            scores, weights, done = np.full(6, -2.0, np.float32), np.ones(6, np.float32), np.zeros(6, bool)
            scores[4], weights[4], done[4] = score, weight, ended
            want = ob.select(x.double().cpu().numpy(), scores, 4, 3, 2, done, None, weights)
            assert want[4]
            check_select(run_select(x, scores, 4, 3, 2, done, None, weights), want)
