"""Positions at the end of what 32 bits hold, and steps beyond the largest."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import tokens as ot
from paper_2411_19114_b200 import binding as pb
from test_gpu_tokens import run_positions

pytestmark = pytest.mark.gpu


def test_the_largest_positions():
    spans = [(128, 1, 1, 1 << 24), ((1 << 24) - 2, 0, 0, 1)]
    total = 128 + (1 << 24) - 1
    want = ot.positions(np.array(spans), [0, 2], [0], [0, total], total)[:, -300:]
    got, status = run_positions(spans, [0, 2], [total - 300], [0, 300], 300)
    assert status == 0 and np.array_equal(got, want) and want.max() == 2**31 - 1


def test_positions_are_formed_modulo_2_to_the_32():
    spans = [(200, 1, 2, 1 << 24), (50, 0, 0, 1)]
    want = ot.positions(np.array(spans), [0, 2], [0], [0, 500], 500)
    got, status = run_positions(spans, [0, 2], [0], [0, 500], 500)
    assert status == 0 and want.max() > 2**31 and np.array_equal(got, want.astype(np.int32))


def test_a_step_beyond_the_largest_counts_as_an_empty_span():
    for step, want in ((1 << 24, [0, 1 << 24, (1 << 24) + 1]), ((1 << 24) + 1, [0, 1, 2])):
        got, status = run_positions([(2, 1, 1, step)], [0, 1], [0], [0, 3], 3)
        assert status == (0 if want[1] > 1 else pb.ERR_BAD_TABLE) and got[0].tolist() == want
