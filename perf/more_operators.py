"""A beam search over an encoder's states behind the preprocessing front-end, as measured work: the
selection of the next beams over beams and vocabulary, the block tables of the beams that go on, the
copies of their open pages, and the attention of the beams' rows to the encoder's states.

``listed()`` names the cases, ``draw()`` makes more of the same ranges, ``prepare()`` builds what a
serving program holds before the call, ``run()`` is one pass: with ``own`` set the library's calls,
otherwise the same operators in elementary torch operations.  ``exact()`` restates in 64 bits what
is computed: the scores of the selection and the attention.  Tables, tokens and copied pages are
whole numbers and unchanged values, which have to be equal.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------------

def listed():
    return [
        # one utterance's beams, a small vocabulary: latency is all there is
        dict(name="select_few", op="select", n=1, beams=4, width=4, vocab=32000, dtype="fp32", masked=False,
             ended=False, weighted=False),
        # a full batch over a large vocabulary: the logits have to be read once
        dict(name="select_many", op="select", n=64, beams=8, width=8, vocab=128000, dtype="bf16", masked=False,
             ended=False, weighted=False),
        # rows that begin at odd addresses, twice as many candidates as beams, a grammar that rules
        # tokens out, ended beams and a weight by length
        dict(name="select_odd", op="select", n=24, beams=5, width=10, vocab=50003, dtype="fp16", masked=True,
             ended=True, weighted=True),
        # two short searches: latency
        dict(name="reorder_few", op="reorder", n=2, beams=4, length=600, page=16),
        # a full batch of long ones
        dict(name="reorder_many", op="reorder", n=128, beams=8, length=8192, page=16),
        # the open pages of a few beams in a small model
        dict(name="copy_few", op="copy", n=4, beams=4, length=600, page=16, layers=6, hk=8, d=64, dtype="fp16",
             order="nhd"),
        # of a full batch, heads outside the slots
        dict(name="copy_many", op="copy", n=64, beams=8, length=500, page=32, layers=12, hk=8, d=128, dtype="bf16",
             order="hnd"),
        # one step of two utterances' beams over a few seconds of states: latency
        dict(name="cross_few", op="cross", n=2, q=4, states=375, hq=8, hk=8, d=64, dtype="fp16", seen=False),
        # a full batch's beams over half a minute of states, a key head per query head: bytes
        dict(name="cross_beams", op="cross", n=64, q=5, states=1500, hq=20, hk=20, d=64, dtype="bf16", seen=False),
        # eight beams of four query heads on each key head: still bytes, 32 rows share them
        dict(name="cross_group", op="cross", n=48, q=8, states=2000, hq=32, hk=8, d=128, dtype="bf16", seen=False),
        # the decoder's prompts of a batch at once: products
        dict(name="cross_prompts", op="cross", n=16, q=448, states=1500, hq=20, hk=20, d=64, dtype="bf16", seen=False),
        # prompts with images among the text: a row sees the patches of the images before it
        dict(name="cross_images", op="cross", n=6, q=701, states=2308, hq=14, hk=2, d=80, dtype="fp16", seen=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["select", "select", "reorder", "copy", "cross", "cross", "cross"])
    beams = rng.randint(1, 10)
    if op == "select":
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        vocab = _log_int(rng, 1000, 200000)
        most = 64 * 8 * 128000 * 2 // (vocab * beams * (4 if dtype == "fp32" else 2))
        return dict(op=op, n=_log_int(rng, 1, max(1, min(128, most))), beams=beams, width=rng.choice([beams, beams, 2 * beams]),
                    vocab=vocab, dtype=dtype, masked=rng.random() < 0.3, ended=rng.random() < 0.4,
                    weighted=rng.random() < 0.3)
    page = rng.choice([16, 32, 64])
    if op == "reorder":
        length = _log_int(rng, 20, 8192)
        return dict(op=op, n=_log_int(rng, 1, max(1, min(1000, 128 * 8 * 512 // (beams * -(-length // page))))),
                    beams=beams, length=length, page=page)
    dtype, d = rng.choice(["bf16", "fp16"]), rng.choice([64, 64, 128, 8 * rng.randint(8, 16)])
    hk = rng.choice([1, 2, 4, 8, 12])
    if op == "copy":
        return dict(op=op, n=_log_int(rng, 1, max(1, 400 // beams)), beams=beams, length=rng.randint(20, 500), page=page,
                    layers=rng.randint(1, 12), hk=min(hk, 8), d=d, dtype=dtype, order=rng.choice(["nhd", "hnd"]))
    while True:
        n, hq = _log_int(rng, 1, 96), hk * rng.choice([1, 1, 1, 2, 4, 7])
        q = beams if rng.random() < 0.6 else _log_int(rng, 11, 1024)
        states = _log_int(rng, 1, 4000)
        if n * states * hk <= 48 * 2000 * 16 and n * q * hq * states * d <= 16 * 448 * 20 * 1500 * 64:
            break
    return dict(op=op, n=n, q=q, states=states, hq=hq, hk=hk, d=d, dtype=dtype, seen=rng.random() < 0.3)


def _rng(case):
    """Lengths are a property of the case; a seed only permutes them."""
    return random.Random(" ".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name"))


def _lengths(case):
    """Tokens in the cache of each request's beams."""
    rng = _rng(case)
    return [case["length"] if i == 0 else rng.randint(max(1, case["length"] // 4), case["length"])
            for i in range(case["n"])]


def _cross_lengths(case):
    """(rows, states) of every request: all beams have a row each, prompts differ in length."""
    rng = _rng(case)
    got = []
    for i in range(case["n"]):
        q = case["q"] if case["q"] <= 10 or i == 0 else rng.randint(max(1, case["q"] // 2), case["q"])
        got.append((q, case["states"] if i == 0 else rng.randint(max(1, case["states"] // 3), case["states"])))
    return got


def _images(rows, states):
    """How many states each row sees where four images lie evenly in the prompt, the first at its start."""
    return [-(-states * min(4, 1 + 4 * i // rows) // 4) for i in range(rows)]


def _ended(case):
    return case["n"] * case["beams"] // 5 if case["ended"] else 0


def work(case):
    n = case["n"]
    if case["op"] == "select":
        rows, wide = n * case["beams"], 4 if case["dtype"] == "fp32" else 2
        live = rows - _ended(case)
        return {"bytes": live * case["vocab"] * wide + (live * (case["vocab"] // 8) if case["masked"] else 0) +
                9 * rows + 13 * n * case["width"], "flops": 4 * live * case["vocab"]}
    if case["op"] == "reorder":
        # the beams' page numbers in and out, lengths, parents, copies
        held = sum(-(-length // case["page"]) for length in _lengths(case)) * case["beams"]
        return {"bytes": 8 * held + 28 * n * case["beams"], "flops": 0}
    if case["op"] == "copy":
        tokens = sum(c for _, _, c in _copies(case))
        return {"bytes": 2 * 2 * case["layers"] * tokens * case["hk"] * case["d"] * 2 + 16 * n * case["beams"],
                "flops": 0}
    hq, hk, d = case["hq"], case["hk"], case["d"]
    rows = sum(q for q, _ in _cross_lengths(case))
    states = sum(s for _, s in _cross_lengths(case))
    pairs = sum(sum(_images(q, s)) if case["seen"] else q * s for q, s in _cross_lengths(case))
    return {"bytes": 2 * 2 * rows * hq * d + 2 * 2 * states * hk * d + 8 * (n + 1), "flops": 4 * d * hq * pairs}


# ---- inputs ---------------------------------------------------------------------------------------

def _parents(case, rng):
    """Beams of every request that its new beams continue: the better ones have more children."""
    b = case["beams"]
    return [[min(int(rng.random() ** 1.7 * b), b - 1) for _ in range(b)] for _ in range(case["n"])]


def _copies(case):
    """(request, new beam, tokens) of every open page that has to be copied: a property of the case."""
    parents = _parents(case, _rng(dict(case, kind="parents")))
    got = []
    for r, length in enumerate(_lengths(case)):
        for i, p in enumerate(parents[r]):
            if length % case["page"] and p in parents[r][:i]:
                got.append((r, i, length % case["page"]))
    return got


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    order = random.Random(int(seed))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"select": _prepare_select, "reorder": _prepare_reorder, "copy": _prepare_copy,
            "cross": _prepare_cross}[case["op"]](dict(case), g, order, ints)


def _prepare_select(s, g, order, ints):
    n, beams, vocab, width = s["n"], s["beams"], s["vocab"], s["width"]
    rows, words = n * beams, -(-vocab // 32)
    # a language model's logits: a broad mass, and a few tokens that stand out
    logits = torch.empty(rows, vocab, device=DEV).normal_(generator=g).mul_(2)
    top = torch.randint(0, vocab, (rows, 20), generator=g, device=DEV)
    logits.scatter_add_(1, top, torch.rand(rows, 20, generator=g, device=DEV).mul_(14))
    s["logits"] = logits.to(DTYPES[s["dtype"]])
    s["scores"] = torch.rand(rows, generator=g, device=DEV).mul_(-12)
    s["done"] = s["done_out"] = s["allowed"] = s["weights"] = None
    s["end"] = vocab // 3
    if s["ended"]:
        ended = torch.randperm(rows, generator=g, device=DEV) < _ended(s)
        s["done"], s["done_out"] = ended.to(torch.uint8), torch.zeros(n, width, dtype=torch.uint8, device=DEV)
    if s["masked"]:  # one token in eight is ruled out
        bits = torch.randint(0, 1 << 32, (3, rows, words), generator=g, device=DEV)
        s["allowed"] = (bits[0] | bits[1] | bits[2]).to(torch.uint32).view(torch.int32)
    if s["weighted"]:  # one over a power of the length
        s["weights"] = torch.randint(5, 40, (rows,), generator=g, device=DEV).float().pow_(-0.6)
    s["tokens"], s["parents"] = (torch.zeros(n, width, dtype=torch.int32, device=DEV) for _ in range(2))
    s["out"] = torch.zeros(n, width, dtype=torch.float32, device=DEV)
    return s


def _beam_tables(s, g, order, ints):
    """Block tables of beams that share pages from the left; the order of the requests and of the pool's
    pages is the seed's."""
    n, beams, page = s["n"], s["beams"], s["page"]
    lengths, parents = _lengths(s), _parents(s, _rng(dict({k: v for k, v in s.items() if k != "name"}, kind="parents")))
    rng = _rng(dict({k: v for k, v in s.items() if k != "name"}, kind="depth"))
    share = [[rng.uniform(1 / 3, 1) for _ in range(beams)] for _ in range(n)]
    at = list(range(n))
    order.shuffle(at)
    lengths, parents, share = ([v[i] for i in at] for v in (lengths, parents, share))
    held = torch.tensor([-(-length // page) for length in lengths], device=DEV)
    width = int(held.max()) + 1
    col = torch.arange(width, device=DEV)
    # beam b has the pages of the beam before up to some full page, from a third of the length on
    full = torch.tensor([length // page for length in lengths], device=DEV)
    depth = (full[:, None] * torch.tensor(share, device=DEV)).long()
    depth[:, 0] = 0
    fresh = (col >= depth[..., None]) & (col < held[:, None, None])
    number = fresh.flatten().cumsum(0).view(n, beams, width) - 1
    for b in range(1, beams):
        number[:, b] = torch.where(col < depth[:, b, None], number[:, b - 1], number[:, b])
    used = int(fresh.sum())
    total = used + n * beams + 7
    pages = torch.randperm(total, generator=g, device=DEV)
    table = torch.where(col < held[:, None, None], pages[number], -1)
    free = torch.full((total,), -1, dtype=torch.int32, device=DEV)
    free[:total - used] = pages[used:]
    s.update(pages=total, table_width=width, table=table.view(n * beams, width).to(torch.int32), free=free,
             free_count=ints([total - used]), parents=ints(parents).flatten(),
             lengths=ints(lengths).repeat_interleave(beams))
    return s


def _prepare_reorder(s, g, order, ints):
    s = _beam_tables(s, g, order, ints)
    rows = s["n"] * s["beams"]
    s.update(table_out=torch.full_like(s["table"], -1), lengths_out=torch.zeros_like(s["lengths"]),
             copies=torch.zeros(rows, 4, dtype=torch.int32, device=DEV), free_left=ints([0]))
    return s


def _prepare_copy(s, g, order, ints):
    s = _beam_tables(s, g, order, ints)
    got = _plain_reorder(s)
    shape = (s["pages"], s["page"], s["hk"], s["d"])
    if s["order"] == "hnd":
        shape = (s["pages"], s["hk"], s["page"], s["d"])
    made = [torch.empty(shape, dtype=DTYPES[s["dtype"]], device=DEV).normal_(generator=g) for _ in range(2 * s["layers"])]
    if s["order"] == "hnd":
        made = [c.transpose(1, 2) for c in made]
    return dict(s, copies=got["copies"], k=made[:s["layers"]], v=made[s["layers"]:])


def _prepare_cross(s, g, order, ints):
    pairs = _cross_lengths(s)
    order.shuffle(pairs)
    dt, hq, hk, d = DTYPES[s["dtype"]], s["hq"], s["hk"], s["d"]
    cu_q, cu_k, seen = [0], [0], []
    for q, k in pairs:
        cu_q.append(cu_q[-1] + q)
        cu_k.append(cu_k[-1] + k)
        seen += _images(q, k)
    tokens = cu_q[-1]
    # keys and values are halves of one projection of the encoder's output
    kv = torch.empty(cu_k[-1], 2, hk, d, dtype=dt, device=DEV).normal_(generator=g)
    s.update(tokens=tokens, max_q=max(q for q, _ in pairs), cu_q=ints(cu_q), cu_k=ints(cu_k), kv=kv,
             seen_of=ints(seen) if s["seen"] else None, scale=d ** -0.5,
             query=torch.randn(tokens, hq, d, generator=g, device=DEV).mul_(2).to(dt),
             out=torch.zeros(tokens, hq, d, dtype=dt, device=DEV))
    return s


# ---- one pass -------------------------------------------------------------------------------------

def run(s):
    return {"select": _run_select, "reorder": _run_reorder, "copy": _run_copy, "cross": _run_cross}[s["op"]](s)


def _handle(s, make):
    """The marshalled call that a serving program keeps beside its buffers (made on first use)."""
    if "call" not in s:
        from paper_2411_19114_b200 import binding

        s["call"] = make(binding)
    return s["call"]


def _workspace(size):
    return torch.zeros(size, dtype=torch.uint8, device=DEV)


def _bits(allowed, vocab):
    """[rows, vocab] truth values of the words' bits."""
    shift = torch.arange(32, dtype=torch.int32, device=DEV)
    return ((allowed[..., None] >> shift) & 1).bool().flatten(1)[:, :vocab]


def _run_select(s):
    n, beams, vocab, width, end = s["n"], s["beams"], s["vocab"], s["width"], s["end"]
    if own:
        _handle(s, lambda b: b.PreparedBeamSelect(
            s["logits"], s["scores"], s["tokens"], s["parents"], s["out"],
            _workspace(b.preba_beam_select_query(n, beams, width, vocab, s["logits"].dtype)), end_token=end, done=s["done"],
            done_out=s["done_out"], allowed=s["allowed"], weights=s["weights"]))()
        got = {"tokens": s["tokens"], "parents": s["parents"], "scores": s["out"]}
        return dict(got, done=s["done_out"]) if s["ended"] else got
    # values next to one another decide, so they are formed in 64 bits
    x = s["logits"].double()
    if s["masked"]:
        x.masked_fill_(~_bits(s["allowed"], vocab), -math.inf)
    top = x.amax(1, keepdim=True)
    x = x.sub_(top)
    value = x.sub_(x.exp().sum(1, keepdim=True).log_()).add_(s["scores"].double()[:, None])
    if s["ended"]:
        ended = s["done"].bool()
        value.masked_fill_(ended[:, None], -math.inf)
        value[:, end] = torch.where(ended, s["scores"].double(), value[:, end])
    rank = value
    if s["weighted"]:
        rank = value * s["weights"].double()[:, None]
    rank, value = rank.view(n, -1), value.view(n, -1)
    rank = rank.clone() if rank is value else rank
    picks, scores = [], []
    for _ in range(width):  # the first of equals each time
        at = rank.argmax(1, keepdim=True)
        picks.append(at)
        scores.append(torch.where(rank.gather(1, at) > -math.inf, value.gather(1, at), -math.inf))
        rank.scatter_(1, at, -math.inf)
    at, scores = torch.cat(picks, 1), torch.cat(scores, 1)
    there = scores > -math.inf  # a request whose beams have all ended has no more candidates than beams
    got = {"tokens": torch.where(there, at % vocab, -1).to(torch.int32),
           "parents": torch.where(there, at // vocab, -1).to(torch.int32), "scores": scores.float()}
    if s["ended"]:
        row = at // vocab + torch.arange(n, device=DEV)[:, None] * beams
        got["done"] = (there & ((s["done"][row] != 0) | (got["tokens"] == end))).to(torch.uint8)
    return got


def _plain_reorder(s):
    n, beams, page, width = s["n"], s["beams"], s["page"], s["table_width"]
    table, lengths = s["table"].view(n, beams, width), s["lengths"].view(n, beams)
    parents = s["parents"].view(n, beams).long()
    held = (lengths + page - 1) // page
    col = torch.arange(width, device=DEV)
    have = col < held[..., None]
    new_len = lengths.gather(1, parents)
    new_held = held.gather(1, parents)
    new = table.gather(1, parents[..., None].expand(-1, -1, width))
    new = torch.where(col < new_held[..., None], new, -1)
    # pages that no new beam holds, once each, in the order of request, column, beam
    gone = have.clone()
    for b in range(beams):
        for i in range(beams):
            gone[:, b] &= new[:, i] != table[:, b]
        for i in range(b):
            gone[:, b] &= ~(have[:, i] & (table[:, i] == table[:, b]))
    flat = gone.transpose(1, 2).flatten()
    number = flat.cumsum(0) - 1
    released = torch.full((flat.numel() + 1,), -1, dtype=torch.int32, device=DEV)
    released.scatter_(0, torch.where(flat, number, flat.numel()), table.transpose(1, 2).flatten())
    n_released = flat.sum()
    # every child but the first needs an open page of its own
    again = torch.zeros(n, beams, dtype=torch.bool, device=DEV)
    for i in range(1, beams):
        again[:, i] = (parents[:, :i] == parents[:, i:i + 1]).any(1)
    copied = (again & (new_len % page != 0)).flatten()
    k = copied.cumsum(0) - 1
    free, count = s["free"], s["free_count"]
    page_of = torch.where(k < n_released, released[k.clamp(0, flat.numel())],
                          free[(count - 1 - (k - n_released)).clamp(0, free.numel() - 1)])
    last = (new_held.flatten().long() - 1).clamp(min=0)[:, None]
    new = new.reshape(n * beams, width)
    source = new.gather(1, last).flatten()
    new.scatter_(1, last, torch.where(copied, page_of, source)[:, None])
    zero = torch.zeros_like(source)
    copies = torch.stack([torch.where(copied, source, 0), torch.where(copied, page_of, 0),
                          torch.where(copied, new_len.flatten() % page, 0), zero], 1)
    # what is released beyond the copies goes on top of the stack
    n_copied = copied.sum()
    place = torch.arange(free.numel(), device=DEV) - count
    from_list = (place + n_copied).clamp(0, flat.numel())
    stack = torch.where((place >= 0) & (place < n_released - n_copied), released[from_list], free)
    left = (count + n_released - n_copied).to(torch.int32)
    return {"table": new, "lengths": new_len.flatten(), "copies": copies.to(torch.int32), "free": stack, "left": left}


def _run_reorder(s):
    if not own:
        return _plain_reorder(s)
    _handle(s, lambda b: b.PreparedBeamPages(
        s["parents"], s["lengths"], s["table"], s["table_out"], s["lengths_out"], s["copies"], s["free"],
        s["free_count"], s["free_left"], s["page"],
        _workspace(b.preba_beam_pages_query(s["n"], s["beams"], s["table_width"])), beams=s["beams"], pages=s["pages"]))()
    return {"table": s["table_out"], "lengths": s["lengths_out"], "copies": s["copies"], "free": s["free"],
            "left": s["free_left"]}


def _run_copy(s):
    if own:
        _handle(s, lambda b: b.PreparedPagesCopy(s["copies"], s["k"], s["v"]))()
        return s["k"], s["v"]
    # rows without a copy repeat another row's
    live = s["copies"][:, 2] > 0
    row = torch.where(live, torch.arange(live.numel(), device=DEV), s["copies"][:, 2].argmax())
    source, to, count = s["copies"][row, 0].long(), s["copies"][row, 1].long(), s["copies"][row, 2]
    slot = torch.arange(s["page"], device=DEV)
    slot = torch.where(slot < count[:, None], slot, 0)
    for c in s["k"] + s["v"]:
        c[to[:, None], slot] = c[source[:, None], slot]
    return s["k"], s["v"]


def _run_cross(s):
    n, hq, hk, d = s["n"], s["hq"], s["hk"], s["d"]
    if own:
        _handle(s, lambda b: b.PreparedCrossAttend(
            s["query"], s["kv"][:, 0], s["kv"][:, 1], s["cu_q"], s["cu_k"], s["out"],
            _workspace(b.preba_cross_attend_query(n, s["tokens"], hq, hk, d)), max_q=s["max_q"], scale=s["scale"],
            seen=s["seen_of"]))()
        return s["out"]
    qm, km, group = s["max_q"], s["states"], hq // hk
    out = torch.zeros(s["tokens"], hq, d, device=DEV)
    i, j = torch.arange(qm, device=DEV), torch.arange(km, device=DEV)
    rows, states = s["cu_q"].diff(), s["cu_k"].diff()
    token = (s["cu_q"][:-1, None] + i).clamp(max=s["tokens"] - 1).long()
    state = (s["cu_k"][:-1, None] + j).clamp(max=s["kv"].shape[0] - 1).long()
    limit = states[:, None].expand(n, qm)
    if s["seen_of"] is not None:
        limit = torch.minimum(limit, s["seen_of"][token])
    step = max(1, (1 << 29) // (qm * hq * km))  # requests at a time, to bound the memory
    for r in range(0, n, step):
        q = s["query"][token[r:r + step]].float().view(-1, qm, hk, group, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
        k, v = (s["kv"][state[r:r + step], c].permute(0, 2, 1, 3).float() for c in (0, 1))
        score = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(-1, hk, group, qm, km)
        hidden = j >= limit[r:r + step, :, None]
        score.masked_fill_(hidden[:, None, None], -math.inf)
        p = score.sub_(score.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
        total = p.sum(-1, keepdim=True)
        part = (p.flatten(2, 3) @ v).view(-1, hk, group, qm, d)
        part = torch.where(total > 0, part / total, 0.0).permute(0, 3, 1, 2, 4).reshape(-1, hq, d)
        valid = (i < rows[r:r + step, None]).flatten()
        # rows behind a request's last go to the place of their clamped token and add nothing
        out.index_add_(0, token[r:r + step].flatten(), part * valid[:, None, None])
    return out.to(s["query"].dtype)


# ---- the definition in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    if case["op"] in ("reorder", "copy"):
        return None  # whole numbers and values as they were: compared for equality
    s = prepare(case, seed)
    if case["op"] == "select":
        vocab, beams, scores = case["vocab"], case["beams"], []
        for r in range(case["n"]):
            rank, value = [], []
            for b in range(r * beams, (r + 1) * beams):
                total = float(s["scores"][b])
                weight = float(s["weights"][b]) if case["weighted"] else 1.0
                if case["ended"] and int(s["done"][b]):
                    v = torch.tensor([total], dtype=torch.float64, device=DEV)
                else:
                    x = s["logits"][b].double()
                    if case["masked"]:
                        x = x[_bits(s["allowed"][b:b + 1], vocab)[0]]
                    v = torch.log_softmax(x, 0) + total
                v = v.topk(min(case["width"], v.numel())).values
                rank.append(v * weight)
                value.append(v)
            none = torch.full((case["width"],), -math.inf, dtype=torch.float64, device=DEV)
            scores.append(torch.cat(value + [none])[torch.cat(rank + [none]).topk(case["width"]).indices])
        got = {"tokens": None, "parents": None, "scores": torch.stack(scores)}
        return dict(got, done=None) if case["ended"] else got
    out = torch.zeros(s["query"].shape, dtype=torch.float64, device=DEV)
    group, cu_q, cu_k = case["hq"] // case["hk"], s["cu_q"].tolist(), s["cu_k"].tolist()
    for r in range(case["n"]):
        k, v = s["kv"][cu_k[r]:cu_k[r + 1]].double().unbind(1)
        t = slice(cu_q[r], cu_q[r + 1])
        key = torch.arange(k.shape[0], device=DEV)
        for h in range(case["hq"]):
            z = s["query"][t, h].double() @ k[:, h // group].t() * s["scale"]
            if s["seen_of"] is not None:
                z = z.masked_fill(key >= s["seen_of"][t, None], -math.inf)
            out[t, h] = torch.softmax(z, -1) @ v[:, h // group]
    return out
