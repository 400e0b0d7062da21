"""Attention whose waits run out, in the checked build, which can have them do so early: the call ends and
reports it, whatever was under way; nothing but the call's own rows is touched; and the next call, on
the same workspace, is right.  This file runs itself in a process of its own (one library a process)."""
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
    from test_gpu_tokens import Step, dev, new_status

    assert pb._LIB_PATH.name == "libpreba_checked.so"
    limit = pb.lib().preba_checked_waits
    limit.restype = None
    # few rows in one piece, split, and in long runs (a run has two tiles at least); many rows claimed, and in a line that is split, both planned by the
    # CTAs and by the planning kernel
    for lengths, hq, hk, d in (([(90, 1), (33, 1)], 8, 2, 64), ([(9000, 1), (200, 1)], 8, 1, 128),
                               ([(1000, 1)] * 64, 16, 8, 128),
                               ([(60 + i % 50, 5) for i in range(500)], 8, 2, 64), ([(6000, 20), (130, 5)], 8, 2, 128),
                               ([(20000, 6)] + [(60, 5)] * 450, 8, 1, 64)):
        step = Step(lengths, hq, hk, d, 16, seed=2)
        want, _, status = step.run()
        assert status == 0
        rows, guard = step.q.shape[0], 64
        ws = torch.zeros(pb.preba_pages_attend_query(len(lengths), rows, hq, hk, d), dtype=torch.uint8, device="cuda")
        whole = torch.full((rows + 2 * guard, hq, d), 3.0, dtype=want.dtype, device="cuda")
        out, status = whole[guard:guard + rows], new_status()
        call = pb.PreparedPagesAttend(step.q, step.k, step.v, dev(step.table), dev(step.cu), dev(step.kv), out, ws,
                                      max_q=step.max_q, scale=step.scale, status=status)

        def run():
            status.zero_()
            call()
            torch.cuda.synchronize()
            assert bool((whole[:guard] == 3).all()) and bool((whole[guard + rows:] == 3).all())
            return int(status.item())

        for waits in (0, 1, 2, 3, 4, 5, 6, 7, 9, 12, 17, 30):
            limit(waits, 1 << 10)
            got = run()
            assert got in (0, pb.ERR_TIMEOUT) and (got or waits > 1), (lengths[0], waits, got)
            if got:
                print("ran out and ended:", lengths[0], waits)
            limit(0, 0)
            out.fill_(3.0)
            assert run() == 0 and torch.equal(out, want), (lengths[0], waits)


if __name__ == "__main__":
    sys.path[:0] = [str(ROOT), str(ROOT / "tests")]
    main()
