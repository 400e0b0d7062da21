"""The serving step where offsets pass 32 bits, and under the checked build of the library."""
from __future__ import annotations

import os
import subprocess
import sys
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import tokens as ot
from paper_2411_19114_b200 import binding as pb

ROOT = Path(__file__).resolve().parent.parent


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 40])
def test_caches_beyond_32_bit_offsets(rows):
    """Two caches of more than 2^32 elements each, of which the last pages are used."""
    page, hk, hq, d = 16, 8, 32, 128
    pages = (1 << 32) // (page * hk * d) + 64
    free, _ = torch.cuda.mem_get_info()
    if free < 5 * pages * page * hk * d:
        pytest.skip("needs 22 GB of device memory")
    k_cache, v_cache = (torch.empty(pages, page, hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv = 70
    table = torch.arange(pages - 5, pages, dtype=torch.int32, device="cuda")[None].contiguous()
    at = torch.arange(kv, device="cuda")
    slots = (table[0, at // page] * page + at % page).to(torch.int32)
    g = torch.Generator(device="cuda").manual_seed(rows)
    k, v = (torch.randn(kv, hk, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(kv, hq, d, generator=g, device="cuda").bfloat16()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    turn = torch.zeros(0, dtype=torch.float64, device="cuda")  # nothing turns: the cache holds what came in
    pos = torch.zeros(3, kv, dtype=torch.int32, device="cuda")
    pb.preba_rope_append(q, k, v, pos, turn, (0, 0, 0), slots, torch.empty_like(q), k_cache, v_cache, status=status)
    assert torch.equal(k_cache[pages - 5:].flatten(0, 1)[:kv], k)
    assert torch.equal(v_cache[pages - 5:].flatten(0, 1)[:kv], v)
    q = q[:rows].contiguous()
    out = torch.empty_like(q)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ws = torch.zeros(pb.preba_pages_attend_query(1, rows, hq, hk, d), dtype=torch.uint8, device="cuda")
    pb.preba_pages_attend(q, k_cache, v_cache, table, ints([0, rows]), ints([kv]), out, ws, max_q=rows,
                          scale=d ** -0.5, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    small = [c[pages - 5:].cpu().double().numpy() for c in (k_cache, v_cache)]
    # slots behind the keys hold whatever the allocation held: no row sees them
    small = [np.where(np.arange(80).reshape(5, page, 1, 1) < kv, c, 0.0) for c in small]
    want, _, spread = ot.attend(q.cpu().double().numpy(), *small, np.arange(5)[None], [0, rows], [kv], d ** -0.5)
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -14) * spread
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= tol)


@pytest.mark.gpu
def test_the_step_runs_clean_under_the_checked_build():
    from paper_2411_19114_b200 import build as pbuild

    pbuild.build(checked=True)
    env = dict(os.environ, PREBA_CHECKED_BUILD="1")
    done = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider",
                           "tests/test_gpu_tokens.py", "-k",
                           "plan or positions or rope or single_tokens or nothing or many_requests or split or out_of_range"],
                          env=env, capture_output=True, text=True, timeout=900, cwd=ROOT)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-2000:]
