"""Attention to packed states whose waits run out, in the checked build, which can have them do so early: the call ends and
reports it, whatever was under way; nothing but the call's own rows is touched; and the next call, on the same workspace, is
right.  This file runs itself in a process of its own (one library a process)."""
from __future__ import annotations

import os
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


@pytest.mark.gpu
def test_waits_that_run_out():
    from paper_2411_19114_b200 import build as pbuild

    pbuild.build(checked=True)
    done = subprocess.run([sys.executable, __file__], env=dict(os.environ, PREBA_CHECKED_BUILD="1"),
                          capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-3000:]
    assert done.stdout.count("ran out and ended") >= 20, done.stdout


def main():
    import torch

    from paper_2411_19114_b200 import binding as pb
    from test_gpu_cross import Step

    assert pb._LIB_PATH.name == "libpreba_checked.so"
    limit = pb.lib().preba_checked_waits
    limit.restype = None
    # few rows: whole pieces, runs that are joined on the spot, one (request, head) over many CTAs; many rows, claimed and in a
    # line, with and without a third tile of scores
    for rows, states, hq, hk, d in (([4, 3], [300, 90], 8, 2, 64), ([5] * 30, [700] * 30, 8, 4, 64), ([16, 2], [30000, 500], 2, 1, 128),
                                    ([8] * 20, [1000] * 20, 32, 8, 128), ([130, 70], [2000, 300], 2, 2, 64),
                                    ([100] * 60, [200] * 60, 8, 8, 64), ([300], [3000], 2, 1, 128)):
        s = Step(rows, states, hq, hk, d, "bf16", seed=2)

        def run():
            s.status.zero_()
            s.call()
            s.out()
            return int(s.status.item())

        assert run() == 0
        want = s.out().clone()
        for waits in (0, 1, 2, 3, 4, 5, 6, 7, 9, 12, 17, 30):
            limit(waits, 1 << 10)
            got = run()
            assert got in (0, pb.ERR_TIMEOUT) and (got or waits > 1), (rows[0], waits, got)
            if got:
                print("ran out and ended:", rows[0], waits)
            limit(0, 0)
            s.whole.fill_(7)
            assert run() == 0 and torch.equal(s.out(), want), (rows[0], waits)


if __name__ == "__main__":
    sys.path[:0] = [str(ROOT), str(ROOT / "tests")]
    main()
