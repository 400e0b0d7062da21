"""Shared memory that a tensor copy fills is written by ordinary stores before that in one place: the limits of the row tiles, which
the attention of many rows keeps in the ring while it plans.  Nothing but a proxy fence of the threads that touched it orders the
two, and a GPU that gets it wrong does so once in a long while: so the order is read from the source."""
from __future__ import annotations

import re
from pathlib import Path

SOURCE = Path(__file__).resolve().parent.parent / "paper_2411_19114_b200" / "csrc" / "preba_attend_tiles.cu"


def body_of(name: str) -> str:
    text = re.sub(r"//[^\n]*", "", SOURCE.read_text())
    at = text.index("{", re.search(rf"\b{name}\s*\(const tiles_args& a, own_plan_t& plan, int32_t\* limits\)", text).end())
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i]
    raise AssertionError(name)


def test_the_limits_are_fenced_off_from_the_copies_that_follow():
    body = body_of("plan_own")
    last_use = [m.start() for m in re.finditer(r"\blimits\[", body)][-1]
    fence = body.find("fence.proxy.async.shared::cta", last_use)
    assert fence > 0 and "__syncthreads()" in body[fence:], "a barrier behind the fence lets the copies begin"
    # every thread reaches the fence: it stands in the function's own block, or under a condition that all share
    before = body[:fence]
    opened = before.count("{") - before.count("}")
    assert opened == 1 or (opened == 2 and re.search(r"if \(limited\)[^;{}]*$|if \(limited\) \{[^{}]*$", before))


def test_limits_are_the_only_thing_that_is_kept_in_the_ring():
    text = re.sub(r"//[^\n]*", "", SOURCE.read_text())
    assert text.count("plan_own<Packed>(a, own, reinterpret_cast<int32_t*>(smem + L::kRing))") == 1
    assert len(re.findall(r"reinterpret_cast<[^>]*>\(smem \+ L::kRing", text)) == 1
