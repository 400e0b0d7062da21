"""The ways in which the attention of many rows is planned: by every CTA for itself (few pairs of row
tiles), by the planning kernel as one line of key tiles, and as claims, longest first."""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_tokens import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 50), (False, 0)])
def test_claims(causal, window):
    # 500 pairs of row tiles on two key heads, none long beside a CTA's share
    rng = np.random.default_rng(1)
    Step([(int(a) + 5, 5) for a in rng.integers(0, 200, 500)], 8, 2, 64, 16, "fp16", seed=1).check(causal, window)


def test_a_line_from_the_planning_kernel():
    # as many pairs, and one request that is far longer than a CTA's share
    rng = np.random.default_rng(2)
    lengths = [(int(a) + 5, 5) for a in rng.integers(0, 90, 450)]
    lengths[200] = (20000, 6)
    Step(lengths, 8, 1, 64, 32, seed=2).check()


@pytest.mark.parametrize("n", [146, 147, 148, 149, 443, 444, 445])
def test_around_the_number_of_pairs_that_a_cta_plans_itself(n):
    rng = np.random.default_rng(n)
    Step([(int(a) + 5, 5) for a in rng.integers(0, 300, n)], 4, 1, 64, 16, seed=n).check()


def test_pairs_of_long_requests_cross_many_ctas():
    Step([(7000, 100), (0, 0), (130, 130), (4000, 33)], 6, 2, 128, 16, seed=5).check()
    Step([(7000, 70), (3, 9)], 4, 4, 64, 64, "fp16", seed=6).check(window=3000)
