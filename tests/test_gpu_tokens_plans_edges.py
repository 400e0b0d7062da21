"""Where the ways to plan the attention of many rows meet, worked out from the GPU's own number of SMs:
the most pairs of row tiles that a CTA plans for itself, more requests than it has threads, more pairs than
the planning kernel takes in one pass, as claims and as a line.  And all of it under the checked build."""
from __future__ import annotations

import os
import subprocess
import sys
from pathlib import Path

import numpy as np
import pytest
import torch

from test_gpu_tokens import Step

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent


def grid():
    return min(160, torch.cuda.get_device_properties(0).multi_processor_count)


def pairs_at_most(n, tokens, group):
    return tokens // (2 * (128 // group)) + n


@pytest.mark.parametrize("off", [-1, 0, 1])
def test_around_the_most_pairs_that_a_cta_plans_for_itself(off):
    # five rows a request, 64 rows a pair: n + 5 n / 64 pairs; a CTA plans fewer than three a CTA itself
    n = next(n for n in range(1, 1000) if pairs_at_most(n, 5 * n, 4) >= 3 * grid()) + off
    assert (pairs_at_most(n, 5 * n, 4) < 3 * grid()) == (off < 0)
    rng = np.random.default_rng(n)
    Step([(int(a) + 5, 5) for a in rng.integers(0, 300, n)], 4, 1, 64, 16, seed=n).check()


@pytest.mark.parametrize("n", [383, 384, 385, 400])
def test_own_plans_with_about_as_many_requests_as_threads(n):
    # 17 rows and a chunk: many rows, few pairs
    rng = np.random.default_rng(n)
    lengths = [(int(a) + 5, 1 + i % 2) for i, a in enumerate(rng.integers(0, 200, n))]
    lengths[n // 2] = (700, 130)
    assert pairs_at_most(n, sum(r for _, r in lengths), 1) < 3 * grid()
    Step(lengths, 1, 1, 64, 16, "fp16", seed=n).check()


@pytest.mark.parametrize("window", [0, 60])
def test_claims_of_more_pairs_than_one_pass(window):
    rng = np.random.default_rng(7)
    Step([(int(a) + 3, 3) for a in rng.integers(0, 150, 2300)], 6, 1, 64, 16, seed=7).check(window=window)


@pytest.mark.parametrize("at", [0, 1500, 2299])
def test_a_line_of_more_pairs_than_one_pass(at):
    rng = np.random.default_rng(8)
    lengths = [(int(a) + 3, 3) for a in rng.integers(0, 150, 2300)]
    lengths[at] = (40000, 3)  # longer than a CTA's share, and in a pass of its own
    Step(lengths, 6, 1, 64, 32, "fp16", seed=8).check()


def test_plans_run_clean_under_the_checked_build():
    if os.environ.get("PREBA_CHECKED_BUILD") == "1":
        pytest.skip("runs itself")
    from paper_2411_19114_b200 import build as pbuild

    pbuild.build(checked=True)
    done = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider",
                           "tests/test_gpu_tokens_plans.py", "tests/test_gpu_tokens_plans_edges.py",
                           "tests/test_gpu_tokens.py", "-k", "plans or chunks or windows or pages_and_orders or not_causal"],
                          env=dict(os.environ, PREBA_CHECKED_BUILD="1"), capture_output=True, text=True, timeout=900,
                          cwd=ROOT)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-2000:]
