"""A beam search over the paged cache by its definitions: selection, block tables of the beams, copies
of open pages, and attention to an encoder's states, written out request by request in 64 bits and in
whole numbers (numpy).  Test infrastructure only; shares no code with the CUDA path."""
from __future__ import annotations

import math

import numpy as np


def select(logits, scores, width, beams, end=-1, done=None, allowed=None, weights=None):
    """(tokens, parents, scores, done) of the best continuations, and whether a row was at fault.  ``allowed``:
    truth values [rows or 1, vocab]."""
    logits = np.asarray(logits, dtype=np.float64)
    rows, vocab = logits.shape
    n = rows // beams
    tokens, parents = np.full((n, width), -1), np.full((n, width), -1)
    out, ended, bad = np.full((n, width), -math.inf), np.zeros((n, width), dtype=bool), False
    for r in range(n):
        offers = []
        for b in range(beams):
            i = r * beams + b
            score, weight = float(scores[i]), 1.0 if weights is None else float(weights[i])
            if math.isnan(score) or score == math.inf or not 0 < weight < math.inf:
                bad = True
                continue
            if score == -math.inf:
                continue
            if done is not None and done[i]:
                offers.append((-weight * score, b, 0.0, end, score, True))
                continue
            seen = np.arange(vocab) if allowed is None else np.flatnonzero(allowed[i if len(allowed) > 1 else 0])
            x = logits[i, seen]
            if np.isnan(x).any() or (x == math.inf).any():
                bad = True
                continue
            if not len(x) or x.max() == -math.inf:
                continue
            top = x.max()
            lse = top + math.log(np.exp(x - top).sum())
            first = np.lexsort((seen, -x))[:width]  # no row has more than `width` of the best
            for v, logit in zip(seen[first], x[first]):
                if logit > -math.inf:
                    value = logit - lse + score
                    offers.append((-weight * value, b, -logit, int(v), value, int(v) == end))
        for k, (_, b, _, v, value, stop) in enumerate(sorted(offers)[:width]):
            tokens[r, k], parents[r, k], out[r, k], ended[r, k] = v, b, value, stop
    return tokens, parents, out, ended, bad


def pages(parents, lengths, table, beams, page, free, count, capacity, total, kept=None):
    """The next block table and what belongs to it.  ``free``: the stack's memory (``capacity`` numbers), of which
    ``count`` are on it, or it is no stack and every request is refused; entries of the table that are not written are -7."""
    table = np.asarray(table)
    rows, width = table.shape
    out, free = np.full((rows, width), -7), np.array(free)
    lengths_out, copies = np.zeros(rows, dtype=np.int64), np.zeros((rows, 4), dtype=np.int64)
    short = False
    bad = no_stack = not 0 <= count <= capacity
    left = count = 0 if no_stack else count
    served = []
    for r in range(rows // beams):
        mine = range(r * beams, (r + 1) * beams)
        held = [-(-int(lengths[i]) // page) for i in mine]
        if no_stack or any(lengths[i] < 0 or h > width or parents[i] >= beams for i, h in zip(mine, held)):
            bad = True
            for i, h in zip(mine, held):
                out[i, :max(0, min(h, width))] = table[i, :max(0, min(h, width))]
            continue
        took = [int(parents[i]) for i in mine]
        alive = {b for b in took if b >= 0}
        gone = []
        for c in range(max(held)):
            have = {int(table[r * beams + b, c]) for b in alive if c < held[b]}
            for b in range(beams):
                number = int(table[r * beams + b, c]) if c < held[b] else None
                if number is None or number in have or (kept is not None and c < kept[r]):
                    continue
                have.add(number)
                if 0 <= number < total:
                    gone.append(number)
                else:
                    bad = True
        needs = [i for i in range(beams) if took[i] >= 0 and took[i] in took[:i]
                 and lengths[r * beams + took[i]] % page]
        if left + len(gone) < len(needs):
            short = True
            for i, h in zip(mine, held):
                out[i, :h] = table[i, :h]
            continue
        left += len(gone) - len(needs)
        served.append((r, took, held, gone, needs))
    released = [g for s in served for g in s[3]]
    supply = released + [int(p) for p in free[:count][::-1]]
    k = 0
    for r, took, held, _, needs in served:
        for i, b in enumerate(took):
            row = r * beams + i
            if b < 0:
                continue
            out[row, :held[b]] = table[r * beams + b, :held[b]]
            lengths_out[row] = lengths[r * beams + b]
            if i in needs:
                out[row, held[b] - 1] = supply[k]
                if 0 <= supply[k] < total:
                    copies[row] = table[r * beams + b, held[b] - 1], supply[k], lengths_out[row] % page, 0
                else:
                    bad = True
                k += 1
    for j, number in enumerate(released[k:]):
        if count + j < capacity:
            free[count + j] = number
        else:
            bad = True
    return dict(table=out, lengths=lengths_out, copies=copies, free=free, left=min(left, capacity), bad=bad, short=short)


def cross_attend(q, k, v, cu_q, cu_k, scale, seen=None):
    """(out, lse, spread): spread is sum p |v| / sum p, what an error of p is multiplied with."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    hq, hk = q.shape[1], k.shape[1]
    out, spread, lse = np.zeros_like(q), np.zeros_like(q), np.full(q.shape[:2], -math.inf)
    for r in range(len(cu_q) - 1):
        for t in range(int(cu_q[r]), int(cu_q[r + 1])):
            states = int(cu_k[r + 1]) - int(cu_k[r])
            if seen is not None:
                states = min(states, int(seen[t]))
            if states <= 0:
                continue
            at = slice(int(cu_k[r]), int(cu_k[r]) + states)
            for h in range(hq):
                z = scale * (k[at, h * hk // hq] @ q[t, h])
                if z.max() == -math.inf:
                    continue
                p = np.exp(z - z.max())
                out[t, h] = p @ v[at, h * hk // hq] / p.sum()
                spread[t, h] = p @ np.abs(v[at, h * hk // hq]) / p.sum()
                lse[t, h] = z.max() + math.log(p.sum())
    return out, lse, spread
