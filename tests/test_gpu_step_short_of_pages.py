"""The example's server where the stack of free pages does not suffice for all requests: a refused
request keeps what it has, and is served when there are pages again."""
from __future__ import annotations

import sys
from pathlib import Path

import numpy as np
import pytest
import torch

from paper_2411_19114_b200 import binding as pb

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))


@pytest.mark.gpu
def test_a_refused_request_keeps_its_tokens_and_pages():
    import image_prompt_step as ex

    server = ex.Server(2, pages=5, width=4)
    spans = torch.zeros((0, 4), dtype=torch.int32, device="cuda")
    begin = torch.zeros(3, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)

    def step(*fresh):
        hidden = torch.randn(sum(fresh), ex.WIDTH, generator=g, device="cuda").bfloat16()
        server.status.zero_()
        server.step(hidden, list(fresh), spans, begin)
        torch.cuda.synchronize()
        return int(server.status.item())

    assert step(ex.PAGE, ex.PAGE) == 0
    assert server.cached.tolist() == [ex.PAGE, ex.PAGE] and int(server.free_count) == 3
    held = server.table.cpu().numpy()[:, :1].copy()
    # two more pages for the first request; the second, which needs two as well, is refused
    assert step(2 * ex.PAGE, ex.PAGE + 1) == pb.ERR_BUFFER_TOO_SMALL
    assert server.cached.tolist() == [3 * ex.PAGE, ex.PAGE] and int(server.free_count) == 1
    # a request without rows keeps its tokens too; the other goes on behind what it has
    assert step(0, 1) == 0
    assert server.cached.tolist() == [3 * ex.PAGE, ex.PAGE + 1] and int(server.free_count) == 0
    table = server.table.cpu().numpy()
    assert np.array_equal(table[:, :1], held) and table[1, 1] >= 0 and table[1, 2] == -1
    pages = np.concatenate([table[0, :3], table[1, :2]])
    assert len(set(pages.tolist())) == 5  # none is held twice
