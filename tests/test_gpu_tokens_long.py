"""Lengths around the largest that a request may have (PREBA_PAGES_MAX_KEYS): places within a request
are 32-bit numbers, so what would pass them is refused and not followed."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import tokens as ot
from paper_2411_19114_b200 import binding as pb
from test_gpu_tokens import Step, check_plan, dev, new_status, run_plan

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


def attend(kv, rows, table, k, v, q, out, window):
    hq, hk, d, n = q.shape[1], k.shape[2], q.shape[2], len(kv)
    ws = torch.zeros(pb.preba_pages_attend_query(n, q.shape[0], hq, hk, d), dtype=torch.uint8, device="cuda")
    status = new_status()
    pb.preba_pages_attend(q, k, v, table, dev(rows * np.arange(n + 1)), dev(kv), out, ws, max_q=rows,
                          scale=d ** -0.5, window=window, status=status)
    torch.cuda.synchronize()
    return int(status.item())


@pytest.mark.parametrize("rows", [1, 30])
def test_attention_at_and_beyond_the_largest_length(rows):
    g = torch.Generator(device="cuda").manual_seed(rows)
    k, v = (torch.randn(4, PAGE, 2, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(2 * rows, 8, 64, generator=g, device="cuda").bfloat16()
    short = torch.tensor([[0, 1, 2], [3, 3, 3]], dtype=torch.int32, device="cuda")
    want = torch.zeros_like(q)
    # a window over the last keys of three pages, and a plain request beside it
    assert attend([3 * PAGE, 100], rows, short, k, v, q, want, 300) == 0
    table = torch.full((2, WIDTH), -1, dtype=torch.int32, device="cuda")
    last = pb.PAGES_MAX_KEYS // PAGE
    table[0, last - 3:last] = short[0]
    table[1, :3] = short[1]
    out = torch.zeros_like(q)
    assert attend([pb.PAGES_MAX_KEYS, 100], rows, table, k, v, q, out, 300) == 0
    assert torch.equal(out, want)
    table[0, last:] = 2
    for kv in (pb.PAGES_MAX_KEYS + 1, 2**31 - 200, 2**31 - 1):
        out = torch.full_like(q, 3.0)
        assert attend([kv, 100], rows, table, k, v, q, out, 300) == pb.ERR_BAD_TABLE
        assert bool((out[:rows] == 3).all()) and torch.equal(out[rows:], want[rows:])
    torch.cuda.empty_cache()
