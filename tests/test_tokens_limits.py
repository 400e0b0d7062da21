"""Limits of the serving step's calls that the host checks."""
from __future__ import annotations

import pytest

from paper_2411_19114_b200 import binding as pb
from test_tokens_boundary import ATTEND, built_library, refused  # noqa: F401


def test_attend_refuses_more_rows_than_a_request_may_have_keys():
    refused("preba_pages_attend", pb.PrebaPagesAttend, ATTEND,
            [dict(tokens=pb.PAGES_MAX_KEYS + 1), dict(tokens=2**31 - 1), dict(tokens=2**32 - 1)])
    for tokens in (pb.PAGES_MAX_KEYS + 1, 2**31 - 1):
        with pytest.raises(pb.PrebaError):
            pb.preba_pages_attend_query(1, tokens, 8, 8, 64)
    assert pb.preba_pages_attend_query(1, pb.PAGES_MAX_KEYS, 8, 8, 64) > 0
