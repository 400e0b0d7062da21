"""The operators of a serving step of a language model behind the preprocessing front-end, as
measured work: pages for the step's tokens, their three-axis positions, the rotation of queries and
keys with the write into the paged cache, and the attention of the new tokens over that cache.

``listed()`` names the cases, ``draw()`` makes more of the same ranges, ``prepare()`` builds what a
serving program holds before the call, ``run()`` is one pass: with ``own`` set the library's calls,
otherwise the same operators in elementary torch operations in 32 bits.  ``exact()`` restates the
two operators whose results are computed numbers in 64 bits, request by request.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
THETA = 1000000.0  # base of the rotary frequencies


# ---- cases ----------------------------------------------------------------------------------------

def listed():
    return [
        # a decoding step of a small batch: one token each, launch latency is all there is
        dict(name="plan_decode", op="plan", kind="decode", n=64, q=1, kv=4096, page=16),
        # a large step that mixes decoding requests with chunks of prompts
        dict(name="plan_mixed", op="plan", kind="mixed", n=1500, q=512, kv=32768, page=32),
        # a batch of prompts of text around the grids of 224-pixel images in 14-pixel patches
        dict(name="positions_prompts", op="positions", kind="prompt", n=48, q=2000, kv=2000, images=4),
        # the same requests later on: one token each, behind their prompts
        dict(name="positions_decode", op="positions", kind="decode", n=256, q=1, kv=5000, images=6),
        # rotation and cache write of one decoding step
        dict(name="rope_decode", op="rope", kind="decode", n=32, q=1, kv=4096, hq=32, hk=8, d=128,
             page=16, dtype="bf16", pairing="half", axes="blocks", order="nhd"),
        # of a step full of prompt chunks
        dict(name="rope_prompts", op="rope", kind="prompt", n=16, q=1024, kv=1024, hq=32, hk=8, d=128,
             page=16, dtype="bf16", pairing="half", axes="turns", order="nhd"),
        # odd token count, seven query heads per key head, neighbouring pairs, heads outside the slots
        dict(name="rope_odd", op="rope", kind="mixed", n=61, q=333, kv=3001, hq=14, hk=2, d=64,
             page=32, dtype="fp16", pairing="next", axes="blocks", order="hnd"),
        # a few decoding requests: latency counts
        dict(name="attend_decode_few", op="attend", kind="decode", n=4, q=1, kv=2048, hq=32, hk=8,
             d=128, page=16, dtype="bf16", causal=True, window=0, order="nhd"),
        # a full decoding batch of very different lengths: the cache has to be read once
        dict(name="attend_decode_many", op="attend", kind="decode", n=128, q=1, kv=8192, hq=32, hk=8,
             d=128, page=64, dtype="bf16", causal=True, window=0, order="nhd"),
        # one chunk of a long prompt over what is cached of it already: few rows, a long axis
        dict(name="attend_chunk", op="attend", kind="chunk", n=1, q=512, kv=30000, hq=32, hk=8,
             d=128, page=16, dtype="bf16", causal=True, window=0, order="nhd"),
        # whole prompts at once: the products dominate
        dict(name="attend_prompts", op="attend", kind="prompt", n=4, q=4096, kv=4096, hq=32, hk=8,
             d=128, page=16, dtype="bf16", causal=True, window=0, order="nhd"),
        # chunks and decoding requests in one step, odd sizes, a sliding window, small heads
        dict(name="attend_mixed", op="attend", kind="mixed", n=37, q=333, kv=3001, hq=14, hk=2,
             d=64, page=32, dtype="fp16", causal=True, window=1000, order="hnd"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "positions", "rope", "rope", "attend", "attend", "attend"])
    kind = rng.choice(["decode", "mixed", "chunk", "prompt"])
    page = rng.choice([16, 32, 64, 128])
    if op == "plan":
        n = _log_int(rng, 1, 2000)
        q = 1 if kind == "decode" else _log_int(rng, 2, max(3, min(8192, 400000 // n)))
        return dict(op=op, kind=kind, n=n, q=q, kv=q if kind == "prompt" else q + _log_int(rng, 16, 32768),
                    page=page)
    if op == "positions":
        n = _log_int(rng, 1, 500)
        q = 1 if kind == "decode" else _log_int(rng, 2, max(3, min(16384, 200000 // n)))
        return dict(op=op, kind=kind, n=n, q=q, kv=q if kind == "prompt" else q + _log_int(rng, 16, 16384),
                    images=rng.randint(0, 8))
    d = rng.choice([64, 128, 128, 8 * rng.randint(8, 16)])
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 2, 4, 5, 7, 8])
    dtype, order = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["nhd", "nhd", "hnd"])
    if op == "rope":
        n = _log_int(rng, 1, 256)
        q = 1 if kind == "decode" else _log_int(rng, 2, max(3, min(8192, 16000 // n)))
        return dict(op=op, kind=kind, n=n, q=q, kv=q if kind == "prompt" else q + _log_int(rng, 16, 8192),
                    hq=hq, hk=hk, d=d // 16 * 16, page=page, dtype=dtype, pairing=rng.choice(["half", "next"]),
                    axes=rng.choice(["blocks", "turns"]), order=order)
    while True:
        n = _log_int(rng, 1, 128)
        q = 1 if kind == "decode" else _log_int(rng, 2, 4096)
        kv = q if kind == "prompt" else q + _log_int(rng, 16, 32768)
        if n * hq * q * kv <= 4 * 32 * 4096 * 4096 and n * kv * hk * d <= 128 * 8192 * 8 * 128:
            break
    return dict(op=op, kind=kind, n=n, q=q, kv=kv, hq=hq, hk=hk, d=d, page=page, dtype=dtype,
                causal=rng.random() < 0.85, window=rng.choice([0, 0, 0, _log_int(rng, 16, 4096)]),
                order=order)


def _lengths(case):
    """(cached, fresh) of every request: a property of the case; a seed only permutes them."""
    rng = random.Random("%(kind)s %(n)d %(q)d %(kv)d" % case)
    n, q, kv = case["n"], case["q"], case["kv"]
    got = []
    for i in range(n):
        kind = case["kind"]
        if kind == "mixed":  # every fourth request has a chunk, the others one token
            kind = "chunk" if i % 4 == 0 else "decode"
        if kind == "decode":
            got.append((_log_int(rng, max(1, kv // 8), max(1, kv - 1)) if i else kv - 1, 1))
        elif kind == "chunk":
            fresh = rng.randint(max(1, q // 2), q) if i else q
            got.append((rng.randint((kv - q) // 2, kv - q) if i else kv - q, fresh))
        else:
            got.append((0, rng.randint(max(1, q // 2), q) if i else q))
    return got


def _spans(case):
    """(t, h, w, step) spans of every request's prompt, and where each request's spans begin.  Text
    has h = w = 0 and t tokens; an image is a grid of patches, a video several with a time step."""
    rng = random.Random("spans %(n)d %(kv)d %(images)d" % case)
    spans, begin = [], [0]
    for _ in range(case["n"]):
        for _ in range(rng.randint(0, case["images"])):
            spans.append((rng.randint(1, 200), 0, 0, 1))
            side = [(1, 16, 16), (1, 24, 17), (1, 9, 31), (4, 8, 8)][rng.randint(0, 3)]
            spans.append((*side, 2 if side[0] > 1 else 1))
        spans.append((rng.randint(1, 300), 0, 0, 1))
        begin.append(len(spans))
    return spans, begin


def work(case):
    pairs = _lengths(case)
    n, tokens = case["n"], sum(f for _, f in pairs)
    if case["op"] == "plan":
        page = case["page"]
        new = sum(-(-(c + f) // page) - -(-c // page) for c, f in pairs)
        # lengths, free pages and the open page of each request in; table entries, slots,
        # positions, row starts and lengths out
        return {"bytes": 4 * (2 * n + new + n) + 4 * (new + 2 * tokens + 2 * n + 2), "flops": 0}
    if case["op"] == "positions":
        return {"bytes": 16 * len(_spans(case)[0]) + 4 * 3 * n + 12 * tokens, "flops": 0}
    hq, hk, d = case["hq"], case["hk"], case["d"]
    if case["op"] == "rope":
        return {"bytes": 2 * 2 * tokens * (hq + 2 * hk) * d + 16 * tokens + 4 * d,
                "flops": 3 * tokens * (hq + hk) * d}
    keys = seen = 0
    for c, f in pairs:
        w = case["window"] or c + f
        if case["causal"]:
            keys += c + f - max(0, c + 1 - w)
            a = min(max(w - c, 0), f)  # rows that see all that is before them: c+1 .. c+a keys
            seen += a * c + a * (a + 1) // 2 + (f - a) * w
        else:
            keys += c + f - max(0, c + 1 - w)
            seen += sum(c + f - max(0, c + i + 1 - w) for i in range(f))
    return {"bytes": 2 * 2 * tokens * hq * d + 2 * 2 * keys * hk * d + 4 * (keys // case["page"] + 3 * n),
            "flops": 4 * d * hq * seen}


# ---- inputs ---------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    order = random.Random(int(seed))
    pairs = _lengths(case)
    order.shuffle(pairs)
    n, tokens = case["n"], sum(f for _, f in pairs)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    starts = [0]
    for _, f in pairs:
        starts.append(starts[-1] + f)
    s = dict(case, tokens=tokens, max_q=max(f for _, f in pairs), max_kv=max(c + f for c, f in pairs),
             cached=ints([c for c, _ in pairs]), fresh=ints([f for _, f in pairs]),
             cu_q=ints(starts), kv_len=ints([c + f for c, f in pairs]))
    if case["op"] == "positions":
        spans, begin = _spans(case)
        s.update(spans=ints(spans), span_begin=ints(begin),
                 out=torch.zeros(3, tokens, dtype=torch.int32, device=DEV))
        return s
    page = case["page"]
    held = [-(-(c if case["op"] == "plan" else c + f) // page) for c, f in pairs]
    need = [-(-(c + f) // page) for c, f in pairs]
    width, total = max(need), sum(need) + sum(need) // 8 + 3  # a pool that is nearly full
    pages = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    # request r holds the next held[r] pages of the shuffled pool; entries behind them are unset
    first = torch.tensor([0] + held[:-1], device=DEV).cumsum(0)[:, None]
    col = torch.arange(width, device=DEV)[None]
    table = torch.where(col < torch.tensor(held, device=DEV)[:, None],
                        pages[(first + col).clamp(max=total - 1)], ints(-1))
    s.update(table=table, pages_total=total, width=width)
    if case["op"] == "plan":
        free = pages[sum(held):].contiguous()
        s.update(free=free, free_count=ints([free.numel()]), cu=torch.zeros(n + 1, dtype=torch.int32, device=DEV),
                 kv=torch.zeros(n, dtype=torch.int32, device=DEV),
                 slots=torch.zeros(tokens, dtype=torch.int32, device=DEV),
                 positions=torch.zeros(tokens, dtype=torch.int32, device=DEV),
                 free_left=torch.zeros(1, dtype=torch.int32, device=DEV))
        return s
    dt, hq, hk, d = DTYPES[case["dtype"]], case["hq"], case["hk"], case["d"]

    def cache(filled):
        shape = (total, page, hk, d) if case["order"] == "nhd" else (total, hk, page, d)
        c = torch.empty(shape, dtype=dt, device=DEV)
        c = c.normal_(generator=g) if filled else c.zero_()
        return c if case["order"] == "nhd" else c.permute(0, 2, 1, 3)

    if case["op"] == "attend":
        s.update(q=torch.randn(tokens, hq, d, generator=g, device=DEV).mul_(2).to(dt), kc=cache(True),
                 vc=cache(True), scale=d ** -0.5, out=torch.zeros(tokens, hq, d, dtype=dt, device=DEV))
        return s
    # one projection's output holds queries, keys and values side by side
    qkv = torch.randn(tokens, hq + 2 * hk, d, generator=g, device=DEV).to(dt)
    row = torch.repeat_interleave(torch.arange(n, device=DEV), s["fresh"].long())
    at = s["cached"][row] + torch.arange(tokens, device=DEV) - s["cu_q"][row]
    slots = table[row, at // page] * page + at % page
    # text has the same position on all axes; a third of the tokens lie on an image's grid
    grid = torch.rand(tokens, generator=g, device=DEV) < 0.33
    back = torch.randint(0, 24, (3, tokens), generator=g, device=DEV)
    pos = (at[None] - torch.where(grid[None], back, 0)).clamp(min=0).to(torch.int32)
    pairs_d = d // 2
    third = pairs_d * 3 // 8
    s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:], slots=slots.to(torch.int32),
             positions=pos, sections=(pairs_d - 2 * (third * 3 // 4), third * 3 // 4, third * 3 // 4),
             inv_freq=THETA ** (-torch.arange(pairs_d, dtype=torch.float64, device=DEV) / pairs_d),
             kc=cache(False), vc=cache(False), q_out=torch.zeros(tokens, hq, d, dtype=dt, device=DEV))
    return s


# ---- one pass -------------------------------------------------------------------------------------

def run(s):
    return {"plan": _run_plan, "positions": _run_positions, "rope": _run_rope,
            "attend": _run_attend}[s["op"]](s)


def _handle(s, make):
    """The marshalled call that a serving program keeps beside its buffers (made on first use)."""
    if "call" not in s:
        from paper_2411_19114_b200 import binding

        s["call"] = make(binding)
    return s["call"]


def _run_plan(s):
    page, tokens, n = s["page"], s["tokens"], s["n"]
    if own:
        _handle(s, lambda b: b.PreparedPagesPlan(
            s["cached"], s["fresh"], s["table"], s["free"], s["free_count"], page, s["cu"], s["kv"],
            s["slots"], s["positions"], s["free_left"]))()
        return {"table": s["table"], "cu": s["cu"], "kv": s["kv"], "slots": s["slots"],
                "positions": s["positions"], "free_left": s["free_left"]}
    cached, fresh = s["cached"], s["fresh"]
    total = cached + fresh
    held = (cached + page - 1) // page
    need = (total + page - 1) // page - held
    cu = torch.cat([cached.new_zeros(1), torch.cumsum(fresh, 0, dtype=torch.int32)])
    first = torch.cumsum(need, 0, dtype=torch.int32) - need
    col = torch.arange(s["width"], dtype=torch.int32, device=DEV)[None]
    # the k-th new page of the step is the k-th from the top of the stack of free pages
    k = s["free_count"] - 1 - (first[:, None] + col - held[:, None])
    new = (col >= held[:, None]) & (col < (held + need)[:, None])
    table = torch.where(new, s["free"][k.clamp(0, s["free"].numel() - 1)], s["table"])
    token = torch.arange(tokens, dtype=torch.int32, device=DEV)
    row = torch.searchsorted(cu[1:], token, right=True).clamp(max=n - 1)
    pos = cached[row] + token - cu[row]
    slots = table[row, pos // page] * page + pos % page
    return {"table": table, "cu": cu, "kv": total, "slots": slots, "positions": pos,
            "free_left": s["free_count"] - need.sum(dtype=torch.int32)}


def _run_positions(s):
    if own:
        _handle(s, lambda b: b.PreparedRopePositions(s["spans"], s["span_begin"], s["cached"], s["cu_q"],
                                                     s["out"]))()
        return s["out"]
    t, h, w, step = s["spans"].unbind(1)
    text = h == 0
    count = torch.where(text, t, t * h * w)  # tokens of a span
    extent = torch.where(text, t, torch.maximum((t - 1) * step + 1, torch.maximum(h, w)))
    zero = count.new_zeros(1)
    at = torch.cat([zero, torch.cumsum(count, 0, dtype=torch.int32)])  # tokens before a span
    place = torch.cat([zero, torch.cumsum(extent, 0, dtype=torch.int32)])  # positions before it
    token = torch.arange(s["tokens"], dtype=torch.int32, device=DEV)
    row = torch.searchsorted(s["cu_q"][1:], token, right=True).clamp(max=s["n"] - 1)
    b0, b1 = s["span_begin"][row], s["span_begin"][row + 1]
    index = s["cached"][row] + token - s["cu_q"][row]  # within the request
    behind = index - (at[b1] - at[b0])  # >= 0: past the prompt, text
    span = torch.searchsorted(at[1:], index + at[b0], right=True).clamp(max=count.numel() - 1)
    rel = index - (at[span] - at[b0])
    base = place[span] - place[b0]
    hw, ww = (h * w)[span].clamp(min=1), w[span].clamp(min=1)
    plain = text[span]
    axes = torch.stack([torch.where(plain, rel, rel // hw * step[span]),
                        torch.where(plain, rel, rel % hw // ww),
                        torch.where(plain, rel, rel % ww)]) + base
    return torch.where(behind >= 0, place[b1] - place[b0] + behind, axes)


def _axis_of_pair(s):
    """Which axis (0 time, 1 height, 2 width) turns each pair of elements."""
    pairs, (a, b, c) = s["d"] // 2, s["sections"]
    j = torch.arange(pairs, device=DEV)
    if s["axes"] == "blocks":
        return (j >= a).long() + (j >= a + b).long()
    return torch.where((j % 3 == 1) & (j // 3 < b), 1, torch.where((j % 3 == 2) & (j // 3 < c), 2, 0))


def _turn(x, cos, sin, pairing):
    if pairing == "half":
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)


def _run_rope(s):
    if own:
        _handle(s, lambda b: b.PreparedRopeAppend(
            s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["sections"], s["slots"], s["q_out"],
            s["kc"], s["vc"], interleaved=s["pairing"] == "next", axes_in_turn=s["axes"] == "turns"))()
        return s["q_out"], s["kc"], s["vc"]
    angle = s["positions"][_axis_of_pair(s)].t().float() * s["inv_freq"].float()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    page, slots, dt = s["page"], s["slots"], s["q"].dtype
    s["kc"][slots // page, slots % page] = _turn(s["k"].float(), cos, sin, s["pairing"]).to(dt)
    s["vc"][slots // page, slots % page] = s["v"]
    return _turn(s["q"].float(), cos, sin, s["pairing"]).to(dt), s["kc"], s["vc"]


def _run_attend(s):
    if own:
        def make(b):
            query = b.preba_pages_attend_query(s["n"], s["tokens"], s["hq"], s["hk"], s["d"])
            ws = torch.zeros(query, dtype=torch.uint8, device=DEV)
            return b.PreparedPagesAttend(s["q"], s["kc"], s["vc"], s["table"], s["cu_q"], s["kv_len"],
                                         s["out"], ws, max_q=s["max_q"], scale=s["scale"],
                                         causal=s["causal"], window=s["window"])
        _handle(s, make)()
        return s["out"]
    n, hq, hk, d, page, qm = s["n"], s["hq"], s["hk"], s["d"], s["page"], s["max_q"]
    group, span = hq // hk, -(-s["max_kv"] // page)
    table = s["table"][:, :span].clamp(min=0).long()
    key = torch.arange(span * page, device=DEV)
    held = (key < s["kv_len"][:, None])[:, None, :, None]
    k = s["kc"][table].flatten(1, 2).permute(0, 2, 1, 3).float()  # [n, hk, keys, d]
    v = s["vc"][table].flatten(1, 2).permute(0, 2, 1, 3).float().masked_fill_(~held, 0.0)
    i = torch.arange(qm, device=DEV)
    fresh = s["cu_q"][1:] - s["cu_q"][:-1]
    token = (s["cu_q"][:-1, None] + i).clamp(max=s["tokens"] - 1).long()
    q = s["q"][token].float().view(n, qm, hk, group, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
    score = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(n, hk, group, qm, span * page)
    at = ((s["kv_len"] - fresh)[:, None] + i)[:, :, None]  # a row's place among the keys
    seen = (key < s["kv_len"][:, None, None]).expand(n, qm, -1)
    if s["causal"]:
        seen = seen & (key <= at)
    if s["window"]:
        seen = seen & (key > at - s["window"])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ v).view(n, hk, group, qm, d)
    out = torch.where(total > 0, out / total, 0.0)
    row = torch.repeat_interleave(torch.arange(n, device=DEV), fresh.long(), output_size=s["tokens"])
    col = torch.arange(s["tokens"], device=DEV) - s["cu_q"][row]
    return out.permute(0, 3, 1, 2, 4)[row, col].reshape(s["tokens"], hq, d).to(s["q"].dtype)


# ---- the definition in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    if case["op"] in ("plan", "positions"):
        return None  # whole numbers: compared for equality
    s = prepare(case, seed)
    if case["op"] == "rope":
        # every pair as a complex number times e^(i position frequency), one axis at a time
        pairs = case["d"] // 2
        a, b, _ = s["sections"]
        axis = [(0 if j < a else 1 if j < a + b else 2) if case["axes"] == "blocks" else
                (j % 3 if j % 3 and j // 3 < s["sections"][j % 3] else 0) for j in range(pairs)]
        freq = [THETA ** (-j / pairs) for j in range(pairs)]
        pos = s["positions"].double()
        turn = torch.stack([torch.polar(torch.ones_like(pos[0]), pos[axis[j]] * freq[j])
                            for j in range(pairs)], -1)[:, None]

        def rotated(x):
            x = x.double()
            if case["pairing"] == "half":
                z = torch.complex(x[..., :pairs], x[..., pairs:]) * turn
                return torch.cat([z.real, z.imag], -1)
            z = torch.view_as_complex(x.reshape(*x.shape[:-1], pairs, 2).contiguous()) * turn
            return torch.view_as_real(z).flatten(-2)

        kc, vc = s["kc"].double(), s["vc"].double()
        page_of, in_page = s["slots"].long() // case["page"], s["slots"].long() % case["page"]
        kc[page_of, in_page] = rotated(s["k"])
        vc[page_of, in_page] = s["v"].double()
        return rotated(s["q"]), kc, vc
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    group = case["hq"] // case["hk"]
    starts, lengths = s["cu_q"].tolist(), s["kv_len"].tolist()
    for r in range(case["n"]):
        t0, t1, kv = starts[r], starts[r + 1], lengths[r]
        rows = s["table"][r, :-(-kv // case["page"])].long()
        k, v = (c[rows].flatten(0, 1)[:kv].double() for c in (s["kc"], s["vc"]))
        first = kv - (t1 - t0)
        for i0 in range(t0, t1, 1024):  # pieces of rows, to bound the memory
            i1 = min(t1, i0 + 1024)
            at = first + torch.arange(i0 - t0, i1 - t0, device=DEV)[:, None]
            key = torch.arange(kv, device=DEV)[None]
            hidden = torch.zeros(i1 - i0, kv, dtype=torch.bool, device=DEV)
            if case["causal"]:
                hidden |= key > at
            if case["window"]:
                hidden |= key <= at - case["window"]
            for h in range(case["hq"]):
                z = s["q"][i0:i1, h].double() @ k[:, h // group].t() * s["scale"]
                p = torch.softmax(z.masked_fill_(hidden, -math.inf), -1)
                out[i0:i1, h] = torch.nan_to_num(p) @ v[:, h // group]
    return out
