"""How the attention of many rows shares its work out where a pair of row tiles has set-up units in the line beside its key tiles
(packed states): csrc/preba_attend_plan.h, compiled as plain C++, against whole numbers without a limit."""
from __future__ import annotations

import random
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2411_19114_b200" / "csrc"
SET_UP = 2
MAIN = r"""
#include "preba_attend_plan.h"
#include <cinttypes>
#include <cstdio>
using namespace preba::attend;
int main() {
  uint64_t a, b, c, d, e;
  while (std::scanf(" %" SCNu64 " %" SCNu64 " %" SCNu64 " %" SCNu64 " %" SCNu64, &a, &b, &c, &d, &e) == 5)
    std::printf("%d\n", int(plans_own(a, uint32_t(b), uint32_t(c), d, uint32_t(e))));
}
"""


@pytest.fixture(scope="module")
def own(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", str(CSRC), "-o", str(at / "main"),
                    str(at / "main.cpp")], check=True)

    def run(lines):
        text = "\n".join(" ".join(str(v) for v in line) for line in lines)
        done = subprocess.run([str(at / "main")], input=text, check=True, capture_output=True, text=True)
        return [int(v) for v in done.stdout.split()]

    return run


def sizes():
    rng = random.Random(4)
    # lines of 2^31 units and a few more or less
    for pairs, heads, grid in ((256, 1, 148), (32, 8, 148), (1, 128, 148), (443, 1, 148), (479, 1, 160), (5, 88, 160)):
        for off in range(-6, 5):
            tiles = 2 ** 31 // (pairs * heads) + off
            for keys in (128 * tiles - 127, 128 * tiles - 1, 128 * tiles, 128 * tiles + 1):
                if keys < 2 ** 31 - 4096:
                    yield pairs, heads, grid, keys
    for _ in range(3000):
        yield rng.randint(1, 500), rng.choice([1, 2, 8, 12]), rng.randint(1, 160), int(2 ** rng.uniform(0, 31))


def test_a_line_that_a_cta_plans_for_itself_can_be_counted(own):
    asked = list(sizes())
    got = own([(*s, SET_UP) for s in asked])
    assert 0 < sum(got) < len(got)
    for (pairs, heads, grid, keys), yes in zip(asked, got):
        units = pairs * heads * (-(-keys // 128) + SET_UP)  # no pair sees more tiles than all states have
        if yes:
            per = max(2, -(-units // grid))
            assert pairs < 480 and pairs * heads < 3 * grid and units <= 2 ** 31 and grid * per < 2 ** 32
        elif pairs < 480 and pairs * heads < 3 * grid:
            assert pairs * heads * (keys // 128 + 2 + SET_UP) > 2 ** 31


def test_without_set_up_nothing_has_changed(own):
    asked = list(sizes())
    want = [int(p < 480 and p * h < 3 * g and p * h * (k // 128 + 2) <= 2 ** 31) for p, h, g, k in asked]
    assert own([(*s, 0) for s in asked]) == want


def test_with_set_up_fewer_lines_are_planned_so_and_none_more(own):
    asked = list(sizes())
    assert all(a <= b for a, b in zip(own([(*s, SET_UP) for s in asked]), own([(*s, 0) for s in asked])))
