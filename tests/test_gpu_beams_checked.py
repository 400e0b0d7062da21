"""The beam search's tests once more under the checked build, whose kernels test their offsets and indices: the status word
stays as the tests want it."""
from __future__ import annotations

import os
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


@pytest.mark.gpu
def test_the_beam_search_runs_clean_under_the_checked_build():
    from paper_2411_19114_b200 import build as pbuild

    pbuild.build(checked=True)
    done = subprocess.run(
        [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "tests/test_gpu_beams.py", "tests/test_gpu_cross.py",
         "tests/test_gpu_speech_beam_step.py", "-k", "not every_warp and not no_longer_a_line and not 1100"],
        env=dict(os.environ, PREBA_CHECKED_BUILD="1"), capture_output=True, text=True, timeout=900, cwd=ROOT)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-3000:]
