"""The serving step behind the preprocessing front-end by its definitions: pages, positions, rotation
and attention, written out request by request and element by element in 64 bits (numpy).  Test
infrastructure only; shares no code with the CUDA path."""
from __future__ import annotations

import math

import numpy as np

MAX_KEYS = 2**31 - 4096  # tokens of one request


def plan(cached, fresh, table, free_pages, free_count, page, tokens):
    """Block table, row starts, key counts, slots, positions and pages left after a step; requests
    that cannot be served get nothing."""
    n = len(cached)
    table = np.array(table, dtype=np.int64)
    slots, positions = np.full(tokens, -1, dtype=np.int64), np.zeros(tokens, dtype=np.int64)
    starts, kv, ok = [0], [], []
    stack = [int(p) for p in free_pages[:free_count]]
    wanted = 0  # pages that the requests so far asked for, served or not
    bad = short = False
    for r in range(n):
        c, f = int(cached[r]), int(fresh[r])
        begin, end = starts[-1], starts[-1] + max(f, 0)
        starts.append(end)
        pages = -(-(c + f) // page)
        if c < 0 or f < 0 or c + f > MAX_KEYS or end > tokens or pages > table.shape[1]:
            bad = True
            kv.append(0)
            continue
        held = -(-c // page)
        need = pages - held
        wanted += need
        if need and wanted > free_count:
            short = True
            kv.append(0)
            continue
        for col in range(held, pages):
            table[r, col] = stack.pop()
        kv.append(c + f)
        for j in range(f):
            positions[begin + j] = c + j
            slots[begin + j] = table[r, (c + j) // page] * page + (c + j) % page
    starts = [min(s, tokens) for s in starts]
    return dict(table=table, cu_q=np.array(starts), kv_len=np.array(kv), slots=slots,
                positions=positions, free_left=len(stack), bad=bad, short=short)


def positions(spans, span_begin, cached, cu_q, tokens):
    """[3, tokens]: every request's whole prompt is laid out, then the step's rows are cut out."""
    out = np.zeros((3, tokens), dtype=np.int64)
    for r in range(len(cached)):
        at, rows = 0, int(cu_q[r + 1]) - int(cu_q[r])
        prompt = []
        for t, h, w, step in np.asarray(spans)[int(span_begin[r]):int(span_begin[r + 1])].tolist():
            if h == 0:
                prompt += [(at + i,) * 3 for i in range(t)]
                at += t
            else:
                grid = [(at + a * step, at + y, at + x) for a in range(t) for y in range(h) for x in range(w)]
                prompt += grid
                if grid:
                    at = 1 + max(max(g) for g in grid)
        while len(prompt) < int(cached[r]) + rows:
            prompt.append((at,) * 3)
            at += 1
        for j in range(rows):
            out[:, int(cu_q[r]) + j] = prompt[int(cached[r]) + j]
    return out


def axis_of_pair(pairs, sections, in_turn):
    if not in_turn:
        return [0] * sections[0] + [1] * sections[1] + [2] * sections[2]
    return [j % 3 if j % 3 and j // 3 < sections[j % 3] else 0 for j in range(pairs)]


def rotate(x, pos, inv_freq, sections, interleaved, in_turn):
    """x [tokens, heads, d] by pos [3, tokens]; elements past the pairs are copied."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    pairs = len(inv_freq)
    for j, axis in enumerate(axis_of_pair(pairs, sections, in_turn)):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
        angle = np.asarray(pos[axis], dtype=np.float64) * float(inv_freq[j])
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y


def attend(q, k_cache, v_cache, table, cu_q, kv_len, scale, causal=True, window=0):
    """(out, lse, spread): spread is sum p |v| / sum p, what an error of p is multiplied with."""
    q, k_cache, v_cache = (np.asarray(a, dtype=np.float64) for a in (q, k_cache, v_cache))
    tokens, hq, d = q.shape
    page, hk = k_cache.shape[1], k_cache.shape[2]
    out, spread = np.zeros_like(q), np.zeros_like(q)
    lse = np.full((tokens, hq), -math.inf)
    for r in range(len(kv_len)):
        kv, first = int(kv_len[r]), int(kv_len[r]) - (int(cu_q[r + 1]) - int(cu_q[r]))
        for t in range(int(cu_q[r]), int(cu_q[r + 1])):
            at = first + t - int(cu_q[r])
            hi = min(kv, at + 1) if causal else kv
            lo = max(0, at - window + 1) if window else 0
            if hi <= lo:
                continue
            key = np.arange(lo, hi)
            pages, within = np.asarray(table)[r][key // page], key % page
            k, v = k_cache[pages, within], v_cache[pages, within]  # [keys, hk, d]
            for h in range(hq):
                z = scale * (k[:, h * hk // hq] @ q[t, h])
                p = np.exp(z - z.max())
                out[t, h] = p @ v[:, h * hk // hq] / p.sum()
                spread[t, h] = p @ np.abs(v[:, h * hk // hq]) / p.sum()
                lse[t, h] = z.max() + math.log(p.sum())
    return out, lse, spread
