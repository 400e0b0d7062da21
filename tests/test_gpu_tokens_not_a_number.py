"""Scores that are not a number: the row's result and its log-sum-exp are not a number either, and
no other row's are, however the row's keys were split over the GPU."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import tokens as ot
from test_gpu_tokens import Step, host64

pytestmark = pytest.mark.gpu

# few rows in one piece and in many, many rows in whole pieces and split
CASES = [([(90, 1), (33, 1)], 8, 2, 64), ([(9000, 1), (200, 1)], 8, 1, 128), ([(200, 70), (40, 9)], 8, 2, 64),
         ([(6000, 20), (130, 5)], 8, 2, 128), ([(60 + i % 50, 5) for i in range(500)], 8, 2, 64)]


def check(step, lost):
    """`lost` [tokens, heads]: the rows whose scores are not all numbers."""
    out, lse, status = step.run()
    assert status == 0
    got, lost = host64(out), np.asarray(lost)
    assert np.isnan(got[lost]).all() and np.isnan(lse[lost]).all()
    k, v = (torch.nan_to_num(c.cpu().double()).numpy() for c in (step.k, step.v))
    want, want_lse, spread = ot.attend(np.nan_to_num(host64(step.q)), k, v, np.maximum(step.table, 0), step.cu,
                                       step.kv, step.scale)
    tol = step.u * np.abs(want) + (step.u + 2.0 ** -14) * spread + 2.0 ** -25 * int(step.kv.max()) * np.abs(v).max()
    assert np.all(np.abs(got - want)[~lost] <= tol[~lost])
    assert np.all(np.abs(lse - want_lse)[~lost] <= 2.0 ** -13)


@pytest.mark.parametrize("lengths,hq,hk,d", CASES)
def test_a_query_that_is_not_a_number(lengths, hq, hk, d):
    s = Step(lengths, hq, hk, d, 16, seed=2)
    lost = np.zeros(s.q.shape[:2], dtype=bool)
    for row, head in ((0, 3), (s.q.shape[0] - 1, hq - 1)):
        s.q[row, head, d - 1] = float("nan")
        lost[row, head] = True
    check(s, lost)


@pytest.mark.parametrize("lengths,hq,hk,d", CASES)
def test_a_key_that_is_not_a_number(lengths, hq, hk, d):
    s = Step(lengths, hq, hk, d, 16, seed=3)
    at = int(s.kv[0]) - 1  # the first request's last key: its last row alone sees it
    s.k[int(s.table[0, at // 16]), at % 16, 0, 0] = float("nan")
    lost = np.zeros(s.q.shape[:2], dtype=bool)
    lost[lengths[0][1] - 1, :hq // hk] = True
    check(s, lost)
