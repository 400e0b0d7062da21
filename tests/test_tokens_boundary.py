"""Host side of include/preba_tokens.h: the header as plain C, struct sizes, and every refusal that
needs no device."""
from __future__ import annotations

import ctypes
import subprocess
from pathlib import Path

import numpy as np
import pytest

from oracle import tokens as ot
from paper_2411_19114_b200 import binding as pb
from paper_2411_19114_b200 import build as pbuild

ROOT = Path(__file__).resolve().parent.parent
STRUCTS = {"preba_pages_plan_t": pb.PrebaPagesPlan, "preba_rope_positions_t": pb.PrebaRopePositions,
           "preba_rope_append_t": pb.PrebaRopeAppend, "preba_pages_attend_t": pb.PrebaPagesAttend}


@pytest.fixture(scope="module", autouse=True)
def built_library():
    pbuild.build()


def test_header_is_plain_c_and_the_binding_has_its_layout(tmp_path):
    src, exe = tmp_path / "use.c", tmp_path / "use"
    lines = []
    for name, struct in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {field}));' for field, _ in struct._fields_]
    src.write_text('#include "preba_tokens.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {'
                   + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", str(ROOT / "include"),
                    "-o", str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for struct in STRUCTS.values():
        want.append(ctypes.sizeof(struct))
        want += [getattr(struct, field).offset for field, _ in struct._fields_]
    assert got == want


def call(name, struct):
    return getattr(pb.lib(), name)(ctypes.byref(struct), None)


def filled(struct, **values):
    """A struct whose pointers are all some aligned address (never followed: every case is refused)."""
    s = struct()
    for name, kind in struct._fields_:
        if kind is ctypes.c_void_p:
            setattr(s, name, 4096)
    for name, value in values.items():
        if isinstance(value, (tuple, list)):
            getattr(s, name)[:] = value
        else:
            setattr(s, name, value)
    return s


def refused(name, struct, good, cases, code=pb.ERR_INVALID_ARG):
    assert getattr(pb.lib(), name)(None, None) == pb.ERR_INVALID_ARG
    for wrong in cases:
        assert call(name, filled(struct, **{**good, **wrong})) == code, wrong


PLAN = dict(free_left=8192, table_stride=4, table_width=4, free_capacity=8, n=2, tokens=8, page_size=16, pages=64)


def test_plan_refuses():
    refused("preba_pages_plan", pb.PrebaPagesPlan, PLAN, [
        {name: None} for name in ("cached", "fresh", "block_table", "free_pages", "free_count", "cu_q", "kv_len",
                                  "slots", "free_left")] + [
        dict(n=0), dict(n=16385), dict(page_size=0), dict(page_size=4), dict(page_size=24), dict(page_size=512),
        dict(pages=2 ** 28), dict(tokens=2 ** 31), dict(table_stride=3), dict(free_left=4096)])


def test_positions_refuse():
    good = dict(axis_stride=8, n_spans=3, n=2, tokens=8)
    refused("preba_rope_positions", pb.PrebaRopePositions, good, [
        {name: None} for name in ("spans", "span_begin", "cached", "cu_q", "positions")] + [
        dict(n=0), dict(tokens=0), dict(axis_stride=7), dict(spans=4104), dict(n_spans=2 ** 31)])


ROPE = dict(q_stride=(256, 64), k_stride=(128, 64), v_stride=(128, 64), q_out_stride=(256, 64),
            cache_stride=(2048, 128, 64), axis_stride=8, sections=(16, 8, 8), tokens=8, heads_q=4, heads_kv=2,
            head_dim=64, rotary_dim=64, pages=4, page_size=16, dtype=pb.F16)


def test_rope_append_refuses():
    refused("preba_rope_append", pb.PrebaRopeAppend, ROPE, [
        {name: None} for name in ("q", "k", "v", "q_out", "k_cache", "v_cache", "positions", "slots",
                                  "inv_freq")] + [
        dict(tokens=0), dict(heads_q=0, heads_kv=0), dict(head_dim=0), dict(head_dim=60), dict(head_dim=136),
        dict(rotary_dim=72), dict(rotary_dim=24, sections=(12, 0, 0)), dict(rotary_dim=80), dict(sections=(16, 8, 9)),
        dict(sections=(8, 12, 12), flags=pb.ROPE_AXES_IN_TURN), dict(dtype=pb.F32), dict(dtype=pb.U8), dict(flags=4),
        dict(q=4104), dict(k_cache=4100), dict(q_stride=(256, 60)), dict(cache_stride=(2048, 129, 64)),
        dict(page_size=20), dict(pages=2 ** 28)])


ATTEND = dict(workspace_bytes=1 << 30, q_stride=(256, 64), out_stride=(256, 64), k_stride=(2048, 128, 64),
              v_stride=(2048, 128, 64), table_stride=4, table_width=4, n=2, tokens=8, max_q=4, heads_q=4,
              heads_kv=2, head_dim=64, pages=4, page_size=16, dtype=pb.BF16, flags=1, scale=0.125)


def test_attend_refuses():
    refused("preba_pages_attend", pb.PrebaPagesAttend, ATTEND, [
        {name: None} for name in ("q", "k_cache", "v_cache", "block_table", "cu_q", "kv_len", "out",
                                  "workspace")] + [
        dict(n=0), dict(n=16385), dict(tokens=0), dict(max_q=0), dict(heads_q=3), dict(heads_kv=0),
        dict(heads_q=129, heads_kv=1), dict(head_dim=0), dict(head_dim=68), dict(head_dim=136), dict(pages=0),
        dict(page_size=12), dict(page_size=4), dict(page_size=512), dict(table_stride=3), dict(dtype=pb.F32),
        dict(flags=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
        dict(q=4104), dict(out=4098), dict(k_stride=(2048, 130, 64)), dict(workspace=4104), dict(window=2 ** 31)])
    refused("preba_pages_attend", pb.PrebaPagesAttend, ATTEND, [dict(workspace_bytes=0)],
            pb.ERR_BUFFER_TOO_SMALL)


def test_attend_query():
    assert pb.preba_pages_attend_query(1, 1, 8, 8, 64) % 16 == 0
    for args in ((0, 1, 8, 8, 64), (1, 0, 8, 8, 64), (1, 1, 8, 3, 64), (1, 1, 8, 8, 60), (1, 1, 0, 8, 64),
                 (1, 1, 8, 8, 136), (16385, 1, 8, 8, 64)):
        with pytest.raises(pb.PrebaError):
            pb.preba_pages_attend_query(*args)


# ---- the definitions themselves -------------------------------------------------------------------

def test_definition_of_the_plan_by_hand():
    got = ot.plan([15, 0], [3, 2], [[9, -1], [-1, -1]], [4, 5, 6], 3, 16, 6)
    assert got["table"].tolist() == [[9, 6], [5, -1]] and got["cu_q"].tolist() == [0, 3, 5]
    assert got["slots"].tolist() == [9 * 16 + 15, 6 * 16, 6 * 16 + 1, 5 * 16, 5 * 16 + 1, -1]
    assert got["free_left"] == 1 and got["kv_len"].tolist() == [18, 2]


def test_definition_of_the_positions_by_hand():
    # two tokens of text, an image of 2 x 3 patches at 2, a video of two frames with step 4 at 5, text
    spans = [(2, 0, 0, 1), (1, 2, 3, 1), (2, 1, 2, 4)]
    got = ot.positions(spans, [0, 3], [0], [0, 14], 14)
    assert got.T.tolist() == [[0, 0, 0], [1, 1, 1], [2, 2, 2], [2, 2, 3], [2, 2, 4], [2, 3, 2], [2, 3, 3],
                              [2, 3, 4], [5, 5, 5], [5, 5, 6], [9, 5, 5], [9, 5, 6], [10, 10, 10], [11, 11, 11]]
    assert np.array_equal(ot.positions(spans, [0, 3], [6], [0, 4], 5), np.pad(got[:, 6:10], ((0, 0), (0, 1))))


def test_definition_of_the_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(0)
    x, y = rng.normal(size=(2, 1, 1, 32))
    inv = 10.0 ** -np.arange(16)
    for inter in (False, True):
        for turns in (False, True):
            sections = (8, 4, 4)
            rot = lambda v, p: ot.rotate(v, np.full((3, 1), p), inv, sections, inter, turns)  # noqa: B023,E731
            assert np.allclose(np.linalg.norm(rot(x, 77)), np.linalg.norm(x), rtol=1e-14)
            # equal positions on all axes: the product of two heads goes by their distance alone
            assert np.allclose(np.sum(rot(x, 1000) * rot(y, 993)), np.sum(rot(x, 7) * rot(y, 0)), rtol=1e-11)
            assert np.array_equal(rot(x, 0), x)


def test_definition_of_attention_in_closed_forms():
    rng = np.random.default_rng(0)
    k, v, q = rng.normal(size=(4, 8, 2, 16)), rng.normal(size=(4, 8, 2, 16)), rng.normal(size=(3, 4, 16))
    table = [[2, 0], [1, -1]]
    # no scores: the mean of the seen values; the log-sum-exp counts them
    out, lse, _ = ot.attend(q * 0, k, v, table, [0, 2, 3], [11, 3], 1.0)
    seq = np.concatenate([v[2], v[0]])
    assert np.allclose(out[0, 0], seq[:10, 0].mean(0)) and np.allclose(out[1, 3], seq[:11, 1].mean(0))
    assert np.allclose(lse, np.log([[10] * 4, [11] * 4, [3] * 4]))
    # a window of one: the row's own value
    out, _, _ = ot.attend(q, k, v, table, [0, 2, 3], [11, 3], 1.0, window=1)
    assert np.allclose(out[1, 2], seq[10, 1])
    # fewer keys than rows: the first row sees nothing
    out, lse, _ = ot.attend(q[:2], k, v, table[:1], [0, 2], [1], 1.0)
    assert np.array_equal(out[0], np.zeros((4, 16))) and np.all(np.isneginf(lse[0])) and np.all(np.isfinite(lse[1]))
