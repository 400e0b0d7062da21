"""Kernels that are set up while the one before still runs: what they may do before they have waited for
it, read from the sources (on a GPU the fault would be two kernels that wait for one another)."""
from __future__ import annotations

import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2411_19114_b200" / "csrc"


def kernels():
    """(file, name, body) of every kernel; a body ends with the first brace in column 0."""
    for path in sorted(CSRC.glob("preba_pages*.cu")) + sorted(CSRC.glob("preba_attend*.cu")):
        for m in re.finditer(r"__global__ void __launch_bounds__\([^)]*\)\s*(\w+)\([^{]*\{\n(.*?)\n\}", path.read_text(), re.S):
            yield path.name, m.group(1), m.group(2)


def test_every_kernel_waits_once_at_the_top_level():
    found = list(kernels())
    assert {name for _, name, _ in found} == {"plan_kernel", "positions_kernel", "append_kernel", "few_rows_kernel",
                                              "tiles_plan_kernel", "tiles_kernel", "tiles_join_kernel"}
    for path, name, body in found:
        assert len(re.findall(r"^  chained_begin\(\);$", body, re.M)) == body.count("chained_begin") == 1, (path, name)


def test_nothing_that_another_kernel_may_need_is_taken_before_the_wait():
    for path, name, body in kernels():
        before = body[:body.index("chained_begin")]
        for taken in ("tcgen05.alloc", "p.status", "report(", "atomic", "tensor_copy(", "plan_own", "find_run",
                      "return"):
            assert taken not in before, (path, name, taken)
    assert any("tcgen05.alloc" in body for _, _, body in kernels())
