"""oracle/beams.py against closed forms, hand-worked cases and brute force."""
from __future__ import annotations

import itertools
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import beams as ob


def test_selection_by_hand():
    # two beams, three tokens; exp of the logits are whole numbers, so that probabilities are fractions
    logits = np.log([[1.0, 2.0, 5.0], [4.0, 4.0, 2.0]])
    scores = np.log([1 / 2, 1 / 4])
    tokens, parents, value, done, bad = ob.select(logits, scores, 4, 2, end=2)
    # 5/16, 2/16 (beam 0), 4/40 twice (beam 1): tokens 0 and 1 tie, the lower comes first
    assert tokens.tolist() == [[2, 1, 0, 1]] and parents.tolist() == [[0, 0, 1, 1]]
    assert np.allclose(np.exp(value), [[5 / 16, 2 / 16, 4 / 40, 4 / 40]], rtol=1e-14)
    assert done.tolist() == [[True, False, False, False]] and not bad
    tokens, parents, value, done, _ = ob.select(logits, scores, 4, 2, end=2, done=[True, False], weights=[0.5, 1.0])
    assert tokens.tolist() == [[2, 0, 1, 2]] and parents.tolist() == [[0, 1, 1, 1]] and done.tolist() == [[True, False, False, True]]
    assert value[0, 0] == pytest.approx(math.log(1 / 2))


def test_selection_is_what_brute_force_finds_in_fractions():
    rng = np.random.default_rng(3)
    for _ in range(30):
        beams, vocab, width = (int(v) for v in rng.integers(1, 5, 3))
        weights = rng.integers(1, 9, (beams, vocab))
        prior = [Fraction(int(v), 64) for v in rng.choice(np.arange(3, 60), beams, replace=False)]
        allowed = rng.random((beams, vocab)) < 0.7
        offers = []
        for b, v in itertools.product(range(beams), range(vocab)):
            if allowed[b, v]:
                total = sum(int(weights[b, u]) for u in range(vocab) if allowed[b, u])
                offers.append((prior[b] * Fraction(int(weights[b, v]), total), b, v))
        best = sorted(offers, key=lambda o: (-o[0], o[1], o[2]))[:width]
        if any(a[0] == b[0] and a[1] != b[1] for a, b in itertools.combinations(offers, 2)):
            continue  # logarithms of equal fractions are equal to a rounding only
        tokens, parents, value, _, _ = ob.select(np.log(weights), [math.log(p) for p in prior], width, beams, allowed=allowed)
        assert [(p, t) for p, t in zip(parents[0], tokens[0])][:len(best)] == [(b, v) for _, b, v in best]
        assert (tokens[0, len(best):] == -1).all() and np.isinf(value[0, len(best):]).all()


def test_rows_that_offer_nothing():
    inf = math.inf
    for row, score, weight, fault in (([0, -inf], -inf, 1, False), ([math.nan, 0], 0, 1, True), ([inf, 0], 0, 1, True),
                                      ([0, 0], math.nan, 1, True), ([0, 0], 0, 0, True), ([-inf, -inf], 0, 1, False)):
        tokens, *_, bad = ob.select([row], [score], 2, 1, weights=[weight])
        assert (tokens == -1).all() and bad == fault
    assert ob.select([[0, -inf]], [0], 2, 1)[0].tolist() == [[0, -1]]


def test_tables_by_hand():
    # pages of 4 slots; one request, three beams of 6 tokens: page 10 is shared, 11, 12, 13 are open
    table = [[10, 11, -1], [10, 12, -1], [10, 13, -1]]
    got = ob.pages([1, 1, 0], [6, 6, 6], table, 3, 4, [20, 21, 0, 0], 2, 4, 30)
    # beam 2 dies: 13 goes to the second child of beam 1; nothing is left for the stack
    assert got["table"][:, :2].tolist() == [[10, 12], [10, 13], [10, 11]] and got["lengths"].tolist() == [6, 6, 6]
    assert got["copies"].tolist() == [[0, 0, 0, 0], [12, 13, 2, 0], [0, 0, 0, 0]] and got["left"] == 2
    # full pages need no copy, and two pages are left over
    got = ob.pages([1, 1, 1], [8, 8, 8], table, 3, 4, [20, 21, 0, 0], 2, 4, 30)
    assert got["left"] == 4 and got["free"].tolist() == [20, 21, 11, 13] and not got["copies"].any()
    # an empty row, and pages that others hold too
    got = ob.pages([-1, 2, 2], [6, 6, 6], table, 3, 4, [20, 21, 0, 0, 0], 2, 5, 30, kept=[2])
    assert got["copies"].tolist() == [[0] * 4, [0] * 4, [13, 21, 2, 0]] and got["left"] == 1 and got["lengths"].tolist() == [0, 6, 6]
    # too few pages: the request stays as it was
    got = ob.pages([0, 0, 0, 1, 1, 1], [6, 6, 6, 8, 8, 8], table + [[1, 2, -1], [1, 3, -1], [1, 4, -1]], 3, 4, [20], 0, 1, 30)
    assert got["left"] == 1 and not got["short"]  # 12 and 13 serve both copies
    got = ob.pages([0, 1, 1], [6, 6, 6], [[10, 11, -1], [10, 12, -1], [10, -1, -1]], 3, 4, [20], 0, 1, 30)
    assert got["bad"] or got["short"]


def test_attention_is_the_library_softmax():
    import torch

    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((5, 4, 8), (9, 2, 8), (9, 2, 8)))
    out, lse, spread = ob.cross_attend(q.numpy(), k.numpy(), v.numpy(), [0, 2, 5], [0, 6, 9], 0.3, seen=[6, 4, 9, 0, 1])
    for t, (a, n) in enumerate(((0, 6), (0, 4), (6, 3), (6, 0), (6, 1))):
        for h in range(4):
            if n == 0:
                assert not out[t, h].any() and lse[t, h] == -math.inf
                continue
            z = 0.3 * k[a:a + n, h // 2] @ q[t, h]
            assert np.allclose(out[t, h], (torch.softmax(z, 0) @ v[a:a + n, h // 2]).numpy(), atol=1e-13)
            assert np.allclose(lse[t, h], torch.logsumexp(z, 0).item())
            assert np.allclose(spread[t, h], (torch.softmax(z, 0) @ v[a:a + n, h // 2].abs()).numpy(), atol=1e-13)
