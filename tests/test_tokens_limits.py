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


def test_attend_refuses_more_pairs_of_row_tiles_than_claims_can_number():
    # 128 query heads on each of 511 key heads: 2^20 rows and up are too many
    wide = dict(heads_q=511 * 128, heads_kv=511, max_q=1, table_width=1, table_stride=1, workspace_bytes=2**63)
    refused("preba_pages_attend", pb.PrebaPagesAttend, ATTEND,
            [dict(wide, tokens=tokens) for tokens in (2**23 + 2**17, 2**30, pb.PAGES_MAX_KEYS)])
