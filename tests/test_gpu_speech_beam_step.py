"""The example that searches with beams behind the audio path, step by step against the definitions: every hypothesis' keys and
values are kept in lists of its own, which follow the beams as whole copies, so that shared pages, copied pages and the
attention over them have to come to the same.

Tolerances as in test_gpu_tokens.py and test_gpu_cross.py (attention) and test_gpu_beams.py (selection); the rotation's, u |out| +
2^-20 (|x| + |y|), comes on top of the scores: keys and queries are taken as the library rotated them.
"""
from __future__ import annotations

import sys
from pathlib import Path

import numpy as np
import pytest

from oracle import beams as ob
from oracle import tokens as ot

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))


@pytest.mark.gpu
@pytest.mark.parametrize("utterances,beams,steps", [(3, 4, 20), (1, 1, 9), (2, 9, 18)])
def test_the_example_matches_the_definitions_step_by_step(utterances, beams, steps):
    import speech_beam_step as ex

    search, traces = ex.run(utterances, beams, steps)
    host = lambda t: t.cpu().double().numpy()  # noqa: E731
    assert int(search.status.item()) == 0
    rows, u = utterances * beams, 2.0 ** -8
    cu_k = search.cu_k.cpu().numpy()
    cross = [host(kv) for kv in search.cross_kv]
    past = [[([], []) for _ in range(rows)] for _ in range(ex.LAYERS)]  # keys and values of every beam
    inv = search.inv_freq.cpu().numpy()
    scores = np.full((utterances, beams), -np.inf)
    scores[:, 0] = 0
    for step, t in enumerate(traces):
        assert np.array_equal(t["scores"].cpu().numpy(), scores.astype(np.float32))
        for layer, (qkv, q, own, asks, seen) in enumerate(t["layers"]):
            qkv, q = host(qkv), host(q)
            rot = ot.rotate(qkv, np.full((3, rows), step), inv, (ex.DIM // 2, 0, 0), False, False)
            assert np.all(np.abs(q - rot[:, :ex.HEADS_Q]) <= u * np.abs(rot[:, :ex.HEADS_Q]) + 2.0 ** -19 * np.abs(qkv).max())
            # the key as the library rounded it, where that is decided by the definition
            key = rot[:, ex.HEADS_Q:ex.HEADS_Q + ex.HEADS_KV]
            value = qkv[:, ex.HEADS_Q + ex.HEADS_KV:]
            for i in range(rows):
                past[layer][i][0].append(key[i])
                past[layer][i][1].append(value[i])
                k, v = np.array(past[layer][i][0]), np.array(past[layer][i][1])
                want, _, spread = ob.cross_attend(q[i:i + 1], k, v, [0, 1], [0, len(k)], ex.DIM ** -0.5)
                # a key is rounded once: a score is off by u sum |q k|, its exponential by as much
                off = u * ex.DIM ** -0.5 * np.abs(q[i]).sum(-1).max() * np.abs(k).max()
                tol = u * np.abs(want) + (u + 2.0 ** -14 + 2 * off) * spread
                assert np.all(np.abs(host(own[i:i + 1]) - want) <= tol), (step, layer, i)
            want, _, spread = ob.cross_attend(host(asks), cross[layer][:, 0], cross[layer][:, 1], np.arange(0, rows + 1, beams),
                                              cu_k, ex.DIM ** -0.5)
            assert np.all(np.abs(host(seen) - want) <= u * np.abs(want) + (u + 2.0 ** -14) * spread + 2.0 ** -25 * 1000)
        tokens, parents, scores, done, bad = ob.select(host(t["logits"]), scores.astype(np.float32).flatten(), beams, beams, ex.END,
                                                       t["done"].cpu().numpy().flatten())
        assert not bad and np.array_equal(t["chosen"].cpu().numpy(), tokens) and np.array_equal(t["parents"].cpu().numpy(), parents)
        assert np.array_equal(t["next_done"].cpu().numpy(), done)
        got = t["next_scores"].cpu().numpy()
        assert np.all(np.abs(got - scores) <= 2.0 ** -18 + 2.0 ** -24 * np.abs(scores))
        scores = got
        for layer in range(ex.LAYERS):
            past[layer] = [tuple(list(part) for part in past[layer][r * beams + parents[r, b]])
                           for r in range(utterances) for b in range(beams)]
    # every page is held by some beam or lies on the stack, once
    table, lengths = search.tables[0].cpu().numpy(), search.lengths.cpu().numpy()
    assert (lengths == steps).all()
    held = {int(p) for i in range(rows) for p in table[i, :-(-lengths[i] // ex.PAGE)]}
    free = search.free.cpu().numpy()[:int(search.free_count)].tolist()
    assert len(free) == len(set(free)) and held.isdisjoint(free) and len(held) + len(free) == search.pages
