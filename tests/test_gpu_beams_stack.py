"""Block tables of beams with a stack of free pages whose count cannot be: no request is served and the stack stays as it is."""
from __future__ import annotations

import numpy as np
import pytest

from paper_2411_19114_b200 import binding as pb
from test_gpu_beams import beam_state, both, run_pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beams", [4, 9])
def test_a_count_that_cannot_be_leaves_the_stack_alone(beams):
    rng = np.random.default_rng(beams)
    lengths, table, free, total = beam_state(rng, 6, beams, 16, 100)
    for parents in (np.full(6 * beams, -1), np.full(6 * beams, 1), np.tile(np.arange(beams), 6)):
        for count in (-1, -2 ** 31, total + 1, 2 ** 31 - 1):
            got, want = both(parents, lengths, table, beams, 16, free, count, total, total)
            assert want["bad"] and want["left"] == 0 and not got["lengths"].any() and not got["copies"].any()
        # an empty stack and a full one are stacks
        both(parents, lengths, table, beams, 16, free, 0, total, total)
    got = run_pages(np.tile(np.arange(beams), 6), lengths, table, beams, 16, np.arange(total), total, total, total)
    assert got["status"] == 0 and got["left"] == total


def test_a_count_above_the_memory_of_the_stack():
    rng = np.random.default_rng(1)
    lengths, table, free, total = beam_state(rng, 3, 2, 16, 60)
    got = run_pages(np.tile([0, 1], 3), lengths, table, 2, 16, free, 2, 1, total)
    assert got["status"] == pb.ERR_BAD_TABLE and got["left"] == 0
