"""How the attention of many rows shares its work out: csrc/preba_attend_plan.h, compiled as plain C++,
against whole numbers without a limit."""
from __future__ import annotations

import random
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2411_19114_b200" / "csrc"
MAIN = r"""
#include "preba_attend_plan.h"
#include <cinttypes>
#include <cstdio>
using namespace preba::attend;
int main() {
  char what;
  uint64_t a, b, c, d;
  while (std::scanf(" %c %" SCNu64 " %" SCNu64 " %" SCNu64 " %" SCNu64, &what, &a, &b, &c, &d) == 5) {
    if (what == 's') {
      const share_t s = share_out(a, uint32_t(b), uint32_t(c), uint32_t(d));
      std::printf("%d %u %u\n", int(s.claim), s.units, s.per);
    } else if (what == 'p') {
      std::printf("%" PRIu64 " 0 0\n", pairs_at_most(uint32_t(a), uint32_t(b), uint32_t(c)));
    } else {
      std::printf("%d 0 0\n", int(plans_own(a, uint32_t(b), uint32_t(c), d)));
    }
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", str(CSRC), "-o", str(at / "main"),
                    str(at / "main.cpp")], check=True)

    def run(lines):
        text = "\n".join(" ".join(str(v) for v in line) for line in lines)
        done = subprocess.run([str(at / "main")], input=text, check=True, capture_output=True, text=True)
        return [tuple(int(v) for v in line.split()) for line in done.stdout.splitlines()]

    return run


def share(total, heads, longest, grid):
    units = total * heads
    if 3 * longest * grid <= units or units > 2**31:
        return 1, 0, 0
    return 0, units, max(2, -(-units // grid))


def test_work_is_counted_past_32_bits(ask):
    # 128 query heads on one key head, 2^20 rows and keys, not causal: 2^19 pairs of 2^13 key tiles
    sizes = [(2**32, 1, 2**13, 148), (2**32 + 5, 1, 2**13, 148), (2**31, 2, 2**13, 148), (2**29, 8, 2**20, 148),
             # one pair whose line would pass what 32 bits count: claimed, although it is long
             (2**24, 200, 2**24, 148), (2**31 + 1, 1, 2**24, 148), (2**31, 1, 2**24, 148), (2**31 - 1, 1, 2**24, 160),
             (0, 8, 0, 148), (1, 1, 1, 148), (13 * 12, 8, 13, 148), (12 * 13, 3, 12, 1)]
    rng = random.Random(1)
    sizes += [(int(2 ** rng.uniform(0, 54)), rng.choice([1, 2, 8, 100]), int(2 ** rng.uniform(0, 24)),
               rng.randint(1, 160)) for _ in range(2000)]
    got = ask([("s", *s) for s in sizes])
    assert got == [share(*s) for s in sizes]
    for (total, heads, _, grid), (claim, units, per) in zip(sizes, got):
        if not claim:  # every run's beginning is a 32-bit number, and the runs cover the line
            assert units == total * heads and (grid - 1) * per + per < 2**32 and grid * per >= units


def test_pairs_are_counted_past_32_bits(ask):
    sizes = [(16384, 2**31 - 4096, 128), (1, 1, 1), (3, 1000, 4), (16384, 2**31 - 4096, 1)]
    assert [g[0] for g in ask([("p", *s, 0) for s in sizes])] == [t // (2 * (128 // g)) + n for n, t, g in sizes]


def test_a_cta_plans_for_itself_only_what_is_sure_to_be_a_line(ask):
    rng = random.Random(2)
    sizes = [(479, 1, 160, 2**31 - 4096), (443, 1, 148, 2**20), (444, 1, 148, 2**20), (479, 1, 160, 10**4),
             (480, 1, 200, 10**4), (1, 1, 148, 2**31 - 4096), (127, 1, 148, 2**31 - 4096), (129, 1, 148, 2**31 - 4096)]
    sizes += [(rng.randint(1, 500), rng.choice([1, 2, 8]), rng.randint(1, 160), int(2 ** rng.uniform(0, 31)))
              for _ in range(2000)]
    for (pairs, heads, grid, keys), (own, _, _) in zip(sizes, ask([("o", *s) for s in sizes])):
        most = -(-keys // 128) + 1  # key tiles of a pair: a first tile that is cut, too
        if own:
            assert pairs < 480 and not share(pairs * most, heads, most, grid)[0] and pairs * heads * most <= 2**31
        elif pairs < 480 and pairs * heads < 3 * grid:
            assert pairs * heads * (keys // 128 + 2) > 2**31
