"""The example that runs the serving step behind the preprocessing, whole prompts first and single
tokens after that, against the definitions of oracle/tokens.py."""
from __future__ import annotations

import sys
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import tokens as ot

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))


@pytest.mark.gpu
def test_the_example_matches_the_definitions_step_by_step():
    import image_prompt_step as ex

    requests, new_tokens = 3, 4
    server, steps = ex.run(requests, new_tokens)
    assert int(server.status.item()) == 0 and len(steps) == 1 + new_tokens
    side, u = 224 // ex.PATCH, 2.0 ** -8
    spans, begin, prompt = [], [0], []
    for r in range(requests):
        spans += [(5 + 7 * r, 0, 0, 1), (1, side, side, 1), (3 + r, 0, 0, 1)]
        begin.append(len(spans))
        prompt.append(8 + 8 * r + side * side)
    table = server.table.cpu().numpy()
    cached, k_all, v_all = np.zeros(requests, dtype=int), [[] for _ in range(requests)], [[] for _ in range(requests)]
    k_cache, v_cache = (c.cpu().double().numpy() for c in (server.layer.k_cache, server.layer.v_cache))
    inv = server.inv_freq.cpu().numpy()
    for step, (hidden, q, out, positions, slots) in enumerate(steps):
        fresh = np.array(prompt if step == 0 else [1] * requests)
        cu = np.concatenate([[0], np.cumsum(fresh)])
        tokens = int(cu[-1])
        want_pos = ot.positions(np.array(spans), begin, cached, cu, tokens)
        assert np.array_equal(positions.cpu().numpy(), want_pos)
        row = np.repeat(np.arange(requests), fresh)
        at = cached[row] + np.arange(tokens) - cu[row]
        assert np.array_equal(slots.cpu().numpy(), table[row, at // ex.PAGE] * ex.PAGE + at % ex.PAGE)
        # the rotation, from the same projection in the library's type
        qkv = (hidden @ server.layer.qkv).view(tokens, -1, ex.DIM).cpu().double().numpy()
        rot = ot.rotate(qkv, want_pos, inv, server.sections, False, False)
        size = np.abs(qkv).max()
        got_q = q.cpu().double().numpy()
        assert np.all(np.abs(got_q - rot[:, :ex.HEADS_Q]) <= u * np.abs(rot[:, :ex.HEADS_Q]) + 2.0 ** -19 * size)
        got_k = k_cache[table[row, at // ex.PAGE], at % ex.PAGE]
        want_k = rot[:, ex.HEADS_Q:ex.HEADS_Q + ex.HEADS_KV]
        assert np.all(np.abs(got_k - want_k) <= u * np.abs(want_k) + 2.0 ** -19 * size)
        assert np.array_equal(v_cache[table[row, at // ex.PAGE], at % ex.PAGE], qkv[:, ex.HEADS_Q + ex.HEADS_KV:])
        # the attention, from the queries and the cache as the library left them
        cached = cached + fresh
        want, _, spread = ot.attend(got_q, k_cache, v_cache, table, cu, cached, ex.DIM ** -0.5)
        tol = u * np.abs(want) + (u + 2.0 ** -14) * spread
        assert np.all(np.abs(out.cpu().double().numpy() - want) <= tol)
    assert np.array_equal(server.kv_len.cpu().numpy(), cached)
