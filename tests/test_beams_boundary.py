"""Host side of include/preba_beams.h: the header as plain C, struct sizes, and every refusal that
needs no device."""
from __future__ import annotations

import ctypes
import subprocess
from pathlib import Path

import pytest
import torch

from paper_2411_19114_b200 import binding as pb
from paper_2411_19114_b200 import build as pbuild

ROOT = Path(__file__).resolve().parent.parent
STRUCTS = {"preba_cross_attend_t": pb.PrebaCrossAttend, "preba_beam_select_t": pb.PrebaBeamSelect, "preba_beam_pages_t": pb.PrebaBeamPages,
           "preba_pages_copy_t": pb.PrebaPagesCopy}


@pytest.fixture(scope="module", autouse=True)
def built_library():
    pbuild.build()


def test_header_is_plain_c_and_the_binding_has_its_layout(tmp_path):
    src, exe = tmp_path / "use.c", tmp_path / "use"
    lines = []
    for name, struct in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {field}));' for field, _ in struct._fields_]
    src.write_text('#include "preba_beams.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {'
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
    """A struct whose pointers are all some aligned address of their own (never followed: every case is refused)."""
    s = struct()
    for k, (name, kind) in enumerate(struct._fields_):
        if kind is ctypes.c_void_p:
            setattr(s, name, 4096 * (k + 1))
    for name, value in values.items():
        if isinstance(value, (tuple, list)):
            getattr(s, name)[:] = value
        else:
            setattr(s, name, value)
    return s


SELECT = dict(workspace_bytes=1 << 40, row_stride=100, allowed_stride=4, n=2, beams=3, width=3, vocab=100, end_token=5,
              dtype=pb.F32)


@pytest.mark.parametrize("change", [
    dict(n=0), dict(beams=0), dict(beams=33), dict(n=5462), dict(width=0), dict(width=65), dict(vocab=0),
    dict(vocab=(1 << 20) + 1, row_stride=1 << 21), dict(dtype=pb.U8), dict(dtype=-1), dict(logits=None), dict(logits=4098),
    dict(scores=None), dict(scores=4097), dict(tokens=None), dict(parents=None), dict(scores_out=None), dict(workspace=None),
    dict(workspace=4104), dict(row_stride=99), dict(row_stride=1 << 38), dict(allowed_stride=3), dict(end_token=-2),
    dict(end_token=100), dict(end_token=-1), dict(weights=4098), dict(allowed=4098), dict(scores_out=8192), dict(tokens=4098),
    dict(parents=4098), dict(scores_out=4098)])
def test_selection_refuses(change):
    assert call("preba_beam_select", filled(pb.PrebaBeamSelect, **{**SELECT, **change})) == pb.ERR_INVALID_ARG


def test_selection_refuses_a_small_workspace():
    need = pb.preba_beam_select_query(2, 3, 3, 100, torch.float32)
    s = filled(pb.PrebaBeamSelect, **{**SELECT, "workspace_bytes": need - 1})
    assert call("preba_beam_select", s) == pb.ERR_BUFFER_TOO_SMALL
    assert pb.lib().preba_beam_select(None, None) == pb.ERR_INVALID_ARG
    with pytest.raises(pb.PrebaError):
        pb.preba_beam_select_query(1, 33, 1, 1, torch.float16)
    with pytest.raises(ValueError):
        pb.preba_beam_select_query(1, 1, 1, 1, torch.float64)


PAGES = dict(workspace_bytes=1 << 40, table_stride=9, table_out_stride=9, table_width=9, free_capacity=50, n=2, beams=3,
             page_size=16, pages=100)


@pytest.mark.parametrize("change", [
    dict(n=0), dict(beams=0), dict(beams=33), dict(n=5462), dict(table_width=0), dict(table_stride=8), dict(table_out_stride=8),
    dict(page_size=4), dict(page_size=24), dict(page_size=512), dict(pages=1 << 27), dict(parents=None), dict(lengths=None),
    dict(table=None), dict(table_out=None), dict(lengths_out=None), dict(copies=None), dict(copies=4104), dict(free_pages=None),
    dict(free_count=None), dict(free_left=None), dict(workspace=None), dict(workspace=4104), dict(table_out=4 * 4096),
    dict(free_left=9 * 4096), dict(lengths_out=2 * 4096), dict(free_capacity=1 << 31),
    dict(table_width=1 << 27, table_stride=1 << 27, table_out_stride=1 << 27),
    dict(n=5000, table_width=1 << 19, table_stride=1 << 19, table_out_stride=1 << 19)])
def test_tables_refuse(change):
    assert call("preba_beam_pages", filled(pb.PrebaBeamPages, **{**PAGES, **change})) == pb.ERR_INVALID_ARG


def test_tables_refuse_a_small_workspace():
    need = pb.preba_beam_pages_query(2, 3, 9)
    s = filled(pb.PrebaBeamPages, **{**PAGES, "workspace_bytes": need - 1})
    assert call("preba_beam_pages", s) == pb.ERR_BUFFER_TOO_SMALL
    assert pb.lib().preba_beam_pages(None, None) == pb.ERR_INVALID_ARG
    with pytest.raises(pb.PrebaError):
        pb.preba_beam_pages_query(1, 0, 5)


COPY = dict(cache_stride=(1024, 64, 64), rows=4, layers=2, heads_kv=1, head_dim=64, pages=10, page_size=16, dtype=pb.F16)


@pytest.mark.parametrize("change", [
    dict(copies=None), dict(copies=4104), dict(k_caches=None), dict(v_caches=None), dict(rows=0), dict(rows=16385),
    dict(layers=0), dict(layers=129), dict(heads_kv=0), dict(heads_kv=65536), dict(head_dim=0), dict(head_dim=60),
    dict(head_dim=136), dict(page_size=12), dict(page_size=512), dict(pages=1 << 28), dict(dtype=pb.F32),
    dict(cache_stride=(1020, 64, 64)), dict(cache_stride=(1 << 38, 64, 64))])
def test_copies_refuse(change):
    pointers = (ctypes.c_void_p * 2)(4096, 8192)
    at = ctypes.cast(pointers, ctypes.c_void_p)
    s = filled(pb.PrebaPagesCopy, **{**COPY, "k_caches": at, "v_caches": at, **change})
    assert call("preba_pages_copy", s) == pb.ERR_INVALID_ARG


def test_copies_refuse_caches_that_are_not_there_or_not_aligned():
    for bad in (0, 4104):
        good, pointers = (ctypes.c_void_p * 2)(4096, 8192), (ctypes.c_void_p * 2)(4096, bad)
        for k, v in ((good, pointers), (pointers, good)):
            s = filled(pb.PrebaPagesCopy, **COPY, k_caches=ctypes.cast(k, ctypes.c_void_p), v_caches=ctypes.cast(v, ctypes.c_void_p))
            assert call("preba_pages_copy", s) == pb.ERR_INVALID_ARG
    assert pb.lib().preba_pages_copy(None, None) == pb.ERR_INVALID_ARG


CROSS = dict(workspace_bytes=1 << 40, q_stride=(512, 64), out_stride=(512, 64), k_stride=(128, 64), v_stride=(128, 64), n=2,
             tokens=6, states=100, max_q=3, heads_q=8, heads_kv=2, head_dim=64, dtype=pb.F16, scale=0.125)


@pytest.mark.parametrize("change", [
    dict(n=0), dict(n=16385), dict(tokens=0), dict(tokens=0x7ffff001), dict(states=0), dict(states=0x7ffff001), dict(max_q=0),
    dict(heads_q=0), dict(heads_q=7), dict(heads_q=258), dict(heads_kv=0), dict(head_dim=0), dict(head_dim=60), dict(head_dim=136),
    dict(dtype=pb.F32), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")),
    dict(q=None), dict(k=None), dict(v=None), dict(cu_q=None), dict(cu_k=None), dict(out=None), dict(workspace=None),
    dict(q=4104), dict(k=4104), dict(v=4104), dict(out=4104), dict(workspace=4104), dict(q_stride=(512, 60)),
    dict(k_stride=(0, 64)), dict(v_stride=(128, 0)), dict(q_stride=(0, 64)), dict(k_stride=(1 << 38, 64)),
    dict(states=0x7f000000, heads_kv=128, heads_q=128), dict(tokens=0x7f000000, heads_q=512, heads_kv=8)])
def test_cross_attention_refuses(change):
    assert call("preba_cross_attend", filled(pb.PrebaCrossAttend, **{**CROSS, **change})) == pb.ERR_INVALID_ARG


def test_cross_attention_refuses_a_small_workspace():
    need = pb.preba_cross_attend_query(2, 6, 8, 2, 64)
    s = filled(pb.PrebaCrossAttend, **{**CROSS, "workspace_bytes": need - 1})
    assert call("preba_cross_attend", s) == pb.ERR_BUFFER_TOO_SMALL
    assert pb.lib().preba_cross_attend(None, None) == pb.ERR_INVALID_ARG
    with pytest.raises(pb.PrebaError):
        pb.preba_cross_attend_query(2, 6, 8, 3, 64)


def test_the_binding_refuses_what_it_cannot_describe():
    t = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype)  # noqa: E731
    f = torch.float32
    good = [t(6, 100, dtype=f), t(6, dtype=f), t(2, 3), t(2, 3), t(2, 3, dtype=f), t(999, dtype=torch.uint8)]
    with pytest.raises(ValueError):  # host tensors
        pb.PreparedBeamSelect(*good)
    with pytest.raises(ValueError):
        pb.PreparedBeamSelect(t(6, 100, dtype=torch.float64), *good[1:])
    h = lambda *shape: torch.zeros(shape, dtype=torch.float16)  # noqa: E731
    with pytest.raises(ValueError):
        pb.PreparedCrossAttend(h(6, 8, 64), h(9, 2, 64), h(9, 2, 64), t(3), t(3), h(6, 8, 64), t(99), 3, 0.1)
    with pytest.raises(ValueError):
        pb.PreparedBeamPages(t(6), t(6), t(6, 9), t(6, 9), t(6), t(6, 4), t(50), t(1), t(1), 16, t(999), 3)
    with pytest.raises(ValueError):
        pb.PreparedPagesCopy(t(6, 4), [], [])
    with pytest.raises(ValueError):
        pb.PreparedPagesCopy(t(6, 4), [t(4, 16, 1, 8, dtype=torch.float16)], [t(4, 16, 1, 8, dtype=torch.float16)])
