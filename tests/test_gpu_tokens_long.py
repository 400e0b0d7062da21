"""Lengths around the largest that a request may have (PREBA_PAGES_MAX_KEYS): places within a request
are 32-bit numbers, so what would pass them is refused and not followed."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import tokens as ot
from paper_2411_19114_b200 import binding as pb
from test_gpu_tokens import check_plan, run_plan

pytestmark = pytest.mark.gpu
PAGE = 256
WIDTH = 2**31 // PAGE + 8  # a row of the table that is long enough for any 31-bit length


@pytest.mark.parametrize("cached,fresh", [
    (2**31 - 1, 10), (2**31 - 1, 0), (pb.PAGES_MAX_KEYS, 1), (pb.PAGES_MAX_KEYS - 3, 4),
    (pb.PAGES_MAX_KEYS - 300, 300), (pb.PAGES_MAX_KEYS, 0), (0, 5)])
def test_plan_refuses_lengths_beyond_the_largest(cached, fresh):
    assert ot.MAX_KEYS == pb.PAGES_MAX_KEYS
    # a plain request before and behind it; pages that the long one holds are page 3, over and over
    table = np.full((3, WIDTH), 3)
    free, c, f = np.arange(10, 18), np.array([5, cached, 20]), np.array([2, fresh, 3])
    want = ot.plan(c, f, table, free, len(free), PAGE, 320)
    assert want["bad"] == (cached + fresh > pb.PAGES_MAX_KEYS) and not want["short"]
    got = run_plan(c, f, table, free, len(free), PAGE, 320)
    assert got["status"] == (pb.ERR_BAD_TABLE if want["bad"] else 0)
    check_plan(got, want)
    torch.cuda.empty_cache()
