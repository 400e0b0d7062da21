"""Refusals that include/preba_beams.h names, beside those of test_beams_boundary.py."""
from __future__ import annotations

import ctypes

import pytest

from paper_2411_19114_b200 import binding as pb
from test_beams_boundary import COPY, CROSS, PAGES, SELECT, built_library, call, filled  # noqa: F401  (a fixture)


def at(struct, name):
    """What filled() puts into this pointer."""
    return getattr(filled(struct), name)


@pytest.mark.parametrize("change", [
    dict(done_out=at(pb.PrebaBeamSelect, "done")), dict(scores_out=at(pb.PrebaBeamSelect, "scores")), dict(allowed_stride=1 << 38),
    dict(end_token=1 << 20), dict(end_token=-2, done=None)])
def test_selection(change):
    assert call("preba_beam_select", filled(pb.PrebaBeamSelect, **{**SELECT, **change})) == pb.ERR_INVALID_ARG


@pytest.mark.parametrize("change", [dict(lengths_out=at(pb.PrebaBeamPages, "lengths")), dict(free_capacity=1 << 31),
                                    dict(free_capacity=(1 << 32) - 1)])
def test_tables(change):
    assert call("preba_beam_pages", filled(pb.PrebaBeamPages, **{**PAGES, **change})) == pb.ERR_INVALID_ARG


@pytest.mark.parametrize("change", [
    dict(q_stride=(1 << 38, 64)), dict(out_stride=(512, 1 << 38)), dict(v_stride=(1 << 38, 64)), dict(dtype=7), dict(scale=-0.0)])
def test_cross_attention(change):
    assert call("preba_cross_attend", filled(pb.PrebaCrossAttend, **{**CROSS, **change})) == pb.ERR_INVALID_ARG


@pytest.mark.parametrize("change", [dict(cache_stride=(1024, 1 << 38, 64)), dict(cache_stride=(1024, 64, 1 << 38)), dict(dtype=9)])
def test_copies(change):
    pointers = ctypes.cast((ctypes.c_void_p * 2)(4096, 8192), ctypes.c_void_p)
    s = filled(pb.PrebaPagesCopy, **{**COPY, "k_caches": pointers, "v_caches": pointers, **change})
    assert call("preba_pages_copy", s) == pb.ERR_INVALID_ARG
