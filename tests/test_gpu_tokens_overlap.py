"""Requests whose rows overlap, which a valid step does not have: reported, and nothing beyond the rows
is touched, however many pairs of row tiles they come to together."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2411_19114_b200 import binding as pb
from test_gpu_tokens import dev, new_status


@pytest.mark.gpu
@pytest.mark.parametrize("n,rows", [(6, 4000), (16384, 1 << 20)])
def test_rows_that_many_requests_share(n, rows):
    # every second request owns all rows (the others' rows run backwards: skipped), with one row of 128
    # query heads to a tile; 16384 requests of 2^20 rows are 2^32 pairs of tiles
    heads, d = 128, 8
    if torch.cuda.mem_get_info()[0] < 6 * rows * heads * d * 2:
        pytest.skip("needs 13 GB of device memory")
    q = torch.ones(rows, heads, d, dtype=torch.bfloat16, device="cuda")
    guard = 1024
    whole = torch.full((rows + 2 * guard, heads, d), 3.0, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(1, 16, 1, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    cu = np.zeros(n + 1, dtype=np.int64)
    cu[1::2] = rows
    ws = torch.zeros(pb.preba_pages_attend_query(n, rows, heads, 1, d), dtype=torch.uint8, device="cuda")
    status = new_status()
    pb.preba_pages_attend(q, k, v, torch.zeros(n, 1, dtype=torch.int32, device="cuda"), dev(cu), dev(np.ones(n)),
                          whole[guard:guard + rows], ws, max_q=rows, scale=1.0, causal=False, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == pb.ERR_BAD_TABLE
    assert bool((whole[guard:guard + rows] == v[0, 0, 0]).all())  # one key: its value
    assert bool((whole[:guard] == 3).all()) and bool((whole[guard + rows:] == 3).all())
    del q, whole, ws
    torch.cuda.empty_cache()
