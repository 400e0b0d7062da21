"""The serving step on the GPU (pages, positions, rotation with the cache write, attention) against
the 64-bit definitions of oracle/tokens.py.

Tolerances, from the arithmetic.  u is the unit roundoff of the 16-bit type (2^-8 bfloat16, 2^-11
binary16).  Rotation: one rounding to the type, and fp32 arithmetic on x and y with an angle that is
off by at most 2^-23 turns: u |out| + 2^-20 (|x| + |y|).  Attention: one rounding of the result,
one rounding of each probability (u sum p|v| / sum p), scores whose fp32 sums are off by at most
2^-15 (twice, for numerator and denominator: 2^-14), and probabilities below the type's normal range,
off by 2^-25 of the largest each: u |out| + (u + 2^-14) spread + 2^-25 keys max|v|.  The
log-sum-exp is off by no more than the scores and a few fp32 roundings: 2^-13.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import tokens as ot
from paper_2411_19114_b200 import binding as pb

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).cuda()


def host(t):
    return t.cpu().numpy()


def host64(t):
    return t.cpu().double().numpy()


def new_status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ---- pages ----------------------------------------------------------------------------------------

def run_plan(cached, fresh, table, free, count, page, tokens, pages=None, positions=True):
    n = len(cached)
    ints = lambda *shape: torch.full(shape, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    t, cu, kv, slots, pos, left, status = (dev(table), ints(n + 1), ints(n), ints(tokens), ints(tokens),
                                           ints(1), new_status())
    free_t = dev(free) if len(free) else torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(2):  # twice: the call changes nothing that it reads
        pb.preba_pages_plan(dev(cached), dev(fresh), t, free_t, dev([count]), page, cu, kv,
                            slots, pos if positions else None, left, pages=pages, status=status)
    torch.cuda.synchronize()
    return dict(table=host(t), cu_q=host(cu), kv_len=host(kv), slots=host(slots),
                positions=host(pos) if positions else None, free_left=int(left.item()),
                status=int(status.item()))


def check_plan(got, want):
    for name in ("table", "cu_q", "kv_len", "slots", "positions"):
        if got[name] is not None:
            assert np.array_equal(got[name], want[name]), name
    assert got["free_left"] == want["free_left"]


@pytest.mark.parametrize("n,page,longest,padding", [
    (1, 16, 1, 0), (1, 8, 700, 3), (3, 256, 600, 0), (33, 16, 40, 1), (511, 32, 9, 5), (512, 64, 70, 0),
    (513, 16, 33, 2), (2000, 16, 20, 0), (16384, 16, 3, 1)])
def test_plan_matches_the_definition(n, page, longest, padding):
    rng = np.random.default_rng(n + page)
    cached, fresh = rng.integers(0, 5 * page, n), rng.integers(0, longest + 1, n)
    fresh[rng.random(n) < 0.2] = 0
    held, need = -(-cached // page), -(-(cached + fresh) // page)
    width = int(need.max()) + 1
    pages = rng.permutation(int(held.sum() + (need - held).sum()) + 4)
    table, at = np.full((n, width), -1), 0
    for r in range(n):
        table[r, :held[r]] = pages[at:at + held[r]]
        at += held[r]
    free = pages[at:]
    tokens = int(fresh.sum()) + padding
    if tokens == 0:
        fresh[0], tokens = 1, 1
    want = ot.plan(cached, fresh, table, free, len(free), page, tokens)
    got = run_plan(cached, fresh, table, free, len(free), page, tokens, pages=len(pages))
    assert got["status"] == 0 and not want["bad"] and not want["short"]
    check_plan(got, want)
    got = run_plan(cached, fresh, table, free, len(free), page, tokens, positions=False)
    check_plan(got, want)


def test_plan_refuses_what_does_not_fit():
    page, table = 16, np.full((6, 4), -1)
    for r, pages in enumerate(([5], [], [6, 7], [], [8], [])):
        table[r, :len(pages)] = pages
    free = np.array([20, 21, 22, 23])
    cached = np.array([10, 0, 32, 0, 3, 0])
    # request 2 takes the stack's last page but one; 3 is too long for what is left, and so is 5
    # behind it, while 4 needs no page
    fresh = np.array([4, 33, 1, 17, 2, 1])
    want = ot.plan(cached, fresh, table, free, 4, page, 64)
    assert want["short"] and list(want["kv_len"]) == [14, 33, 33, 0, 5, 0]
    got = run_plan(cached, fresh, table, free, 4, page, 64)
    assert got["status"] == pb.ERR_BUFFER_TOO_SMALL
    check_plan(got, want)
    # a row of the table that is too short, negative lengths, rows beyond the token arrays
    for c, f, tokens in (([10, 0, 32, 0, 3, 0], [4, 65, 1, 2, 2, 1], 80),
                         ([10, -1, 32, 0, 3, 0], [4, 3, 1, -2, 2, 1], 64),
                         ([10, 0, 32, 0, 3, 0], [4, 3, 1, 2, 2, 1], 9)):
        want = ot.plan(np.array(c), np.array(f), table, free, 4, page, tokens)
        assert want["bad"]
        got = run_plan(c, f, table, free, 4, page, tokens)
        assert got["status"] == pb.ERR_BAD_TABLE
        check_plan(got, want)
    # an open page that the cache does not have; an empty stack; a count beyond the stack
    got = run_plan([10], [4], [[77]], [1], 1, page, 4, pages=50)
    assert got["status"] == pb.ERR_BAD_TABLE and list(got["slots"]) == [-1] * 4
    got = run_plan([10], [9], [[7, -1]], [], 0, page, 9)
    assert got["status"] == pb.ERR_BUFFER_TOO_SMALL and got["free_left"] == 0
    got = run_plan([10], [9], [[7, -1]], [3], 2, page, 9)
    assert got["status"] == pb.ERR_BAD_TABLE and list(got["kv_len"]) == [0]


# ---- positions ------------------------------------------------------------------------------------

def run_positions(spans, begin, cached, cu, tokens):
    out = torch.full((3, tokens + 5), -7, dtype=torch.int32, device="cuda")[:, :tokens]
    status = new_status()
    spans = np.asarray(spans, dtype=np.int64).reshape(-1, 4)
    pb.preba_rope_positions(dev(spans) if len(spans) else torch.zeros((0, 4), dtype=torch.int32, device="cuda"),
                            dev(begin), dev(cached), dev(cu), out, status=status)
    torch.cuda.synchronize()
    return host(out), int(status.item())


@pytest.mark.parametrize("n,most,rows,padding", [(1, 0, 1, 0), (1, 3, 500, 4), (7, 40, 300, 0),
                                                 (40, 5, 1, 0), (300, 3, 70, 9), (2, 100, 4000, 1)])
def test_positions_match_the_definition(n, most, rows, padding):
    rng = np.random.default_rng(n * 100 + most)
    spans, begin = [], [0]
    for _ in range(n):
        for _ in range(rng.integers(0, most + 1)):
            kind = rng.integers(0, 4)
            spans.append([(int(rng.integers(0, 40)), 0, 0, 1), (1, 16, 16, 1), (1, 3, 11, 1),
                          (int(rng.integers(1, 5)), 2, 5, int(rng.integers(1, 9)))][kind])
        begin.append(len(spans))
    fresh = rng.integers(0 if n > 1 else 1, rows + 1, n)
    cached = rng.integers(0, 200, n)
    cu = np.concatenate([[0], np.cumsum(fresh)])
    tokens = int(cu[-1]) + padding
    if tokens == 0:
        pytest.skip("no rows drawn")
    got, status = run_positions(spans, begin, cached, cu, tokens)
    assert status == 0
    assert np.array_equal(got, ot.positions(np.array(spans).reshape(-1, 4), begin, cached, cu, tokens))


def test_positions_skip_what_is_out_of_range():
    # a span with a negative member and one without width count as empty
    got, status = run_positions([(2, 0, 0, 1), (1, -3, 4, 1), (1, 3, 0, 1), (2, 0, 0, 1)], [0, 4], [0], [0, 5], 5)
    assert status == pb.ERR_BAD_TABLE and np.array_equal(got, np.tile(np.arange(5), (3, 1)))
    # spans beyond the table, rows that fall
    got, status = run_positions([(2, 0, 0, 1)], [0, 9, 1], [0, 0], [0, 2, 4], 4)
    assert status == pb.ERR_BAD_TABLE and np.array_equal(got[0], [0, 0, 0, 0])
    got, status = run_positions([(2, 0, 0, 1)], [0, 1, 1], [0, 0], [0, 9, 3], 4)
    assert status == pb.ERR_BAD_TABLE


# ---- rotation and cache write ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens,hq,hk,d,rotary,page,inter,turns,order", [
    (1, 32, 8, 128, 128, 16, False, False, "nhd"), (5, 4, 4, 64, 64, 8, True, True, "hnd"),
    (3, 7, 1, 72, 64, 16, False, True, "nhd"), (130, 14, 2, 64, 32, 32, True, False, "hnd"),
    (9, 5, 5, 8, 0, 16, False, False, "nhd"), (33, 1, 1, 112, 96, 256, False, True, "hnd"),
    (257, 16, 2, 128, 64, 64, True, True, "nhd"), (4, 3, 3, 40, 16, 16, False, False, "nhd")])
def test_rope_append_matches_the_definition(dtype, tokens, hq, hk, d, rotary, page, inter, turns, order):
    dt, u = DTYPES[dtype]
    rng = np.random.default_rng(tokens + d)
    pages = tokens // page + 3
    qkv = torch.tensor(rng.normal(size=(tokens, hq + 2 * hk, d + 8))).to(dt).cuda()[:, :, :d]
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    shape = (pages, page, hk, d) if order == "nhd" else (pages, hk, page, d)
    caches = [torch.tensor(rng.normal(size=shape)).to(dt).cuda() for _ in range(2)]
    if order == "hnd":
        caches = [c.permute(0, 2, 1, 3) for c in caches]
    pos = rng.integers(0, 100000, (3, tokens))
    pos[:, 0] = (1 << 24, 0, 1)
    slots = rng.permutation(pages * page)[:tokens]
    if tokens > 2:
        slots[1] = -1
    pairs = rotary // 2
    inv = 10000.0 ** (-np.arange(pairs) / max(1, pairs))
    part = pairs // 4
    sections = (pairs - 2 * part, part, part)
    want_k, want_v = host64(caches[0]), host64(caches[1])
    rot = lambda x: ot.rotate(host64(x), pos, inv, sections, inter, turns)  # noqa: E731
    size = lambda x: np.abs(host64(x)) + np.abs(host64(x)).max()  # noqa: E731
    for t, s in enumerate(slots):
        if s >= 0:
            want_k[s // page, s % page] = rot(k)[t]
            want_v[s // page, s % page] = host64(v)[t]
    want_q, q_size = rot(q), size(q)
    out, status = torch.zeros_like(q, memory_format=torch.contiguous_format), new_status()
    pb.preba_rope_append(q, k, v, dev(pos), dev(inv, torch.float64), sections, dev(slots), out, *caches,
                         interleaved=inter, axes_in_turn=turns, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert np.all(np.abs(host64(out) - want_q) <= u * np.abs(want_q) + 2.0 ** -20 * q_size)
    got_k = host64(caches[0])
    assert np.all(np.abs(got_k - want_k) <= u * np.abs(want_k) + 2.0 ** -20 * (np.abs(want_k) + 8))
    assert np.array_equal(host64(caches[1]), want_v)


def test_rope_append_in_place_turns_by_one_row():
    rng = np.random.default_rng(3)
    x = torch.tensor(rng.normal(size=(6, 4, 64))).to(torch.float16).cuda()
    k = torch.tensor(rng.normal(size=(6, 2, 64))).to(torch.float16).cuda()
    cache = [torch.zeros(2, 16, 2, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
    inv = 10000.0 ** (-np.arange(32) / 32)
    pos = np.tile(np.arange(6) * 1000, (3, 1))
    want = ot.rotate(host64(x), pos, inv, (16, 8, 8), False, False)
    size = np.abs(host64(x)).max()
    pb.preba_rope_append(x, k, k, dev(pos[:1]).expand(3, 6), dev(inv, torch.float64), (16, 8, 8),
                         dev(np.arange(6)), x, *cache)
    assert np.all(np.abs(host64(x) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -19 * size)


def test_rope_append_leaves_out_slots_beyond_the_cache():
    x = torch.ones(3, 1, 64, dtype=torch.float16, device="cuda")
    cache = [torch.zeros(1, 16, 1, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
    status = new_status()
    pb.preba_rope_append(x, x, x, dev(np.zeros((3, 3))), dev(np.ones(32), torch.float64), (32, 0, 0),
                         dev([2, 16, 5000]), torch.empty_like(x), *cache, status=status)
    assert int(status.item()) == pb.ERR_BAD_TABLE
    assert float(cache[0].sum()) == 64 and float(cache[1][0, 2].sum()) == 64


# ---- attention ------------------------------------------------------------------------------------

class Step:
    """A step's cache, table and queries on the GPU; what no row may see is NaN."""

    def __init__(self, lengths, hq, hk, d, page, dtype="bf16", order="nhd", seed=0, width=None,
                 first_seen=None, scale_q=2.0):
        dt, self.u = DTYPES[dtype]
        rng = np.random.default_rng(seed)
        kv, rows = [a for a, _ in lengths], [b for _, b in lengths]
        n, need = len(kv), [-(-a // page) for a in kv]
        total = sum(need) + 3
        perm = rng.permutation(total)
        self.width = width or max(1, max(need))
        table, at = np.full((n, self.width), -1), 0
        shape = (total, page, hk, d) if order == "nhd" else (total, hk, page, d)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=dt, device="cuda") for _ in range(2))
        if order == "hnd":
            self.k, self.v = self.k.permute(0, 2, 1, 3), self.v.permute(0, 2, 1, 3)
        for r in range(n):
            table[r, :need[r]] = perm[at:at + need[r]]
            at += need[r]
            key = np.arange(first_seen[r] if first_seen else 0, kv[r])
            for c in (self.k, self.v):
                values = torch.tensor(rng.normal(size=(len(key), hk, d))).to(dt).cuda()
                c[dev(table[r, key // page], torch.long), dev(key % page, torch.long)] = values
            if first_seen:  # pages that no row sees need not be there
                table[r, :first_seen[r] // page] = -1 - rng.integers(0, 1000)
        self.table, self.kv, self.cu = table, np.array(kv), np.concatenate([[0], np.cumsum(rows)])
        self.q = torch.tensor(rng.normal(size=(int(self.cu[-1]), hq, d)) * scale_q).to(dt).cuda()
        self.scale, self.max_q, self.d = d ** -0.5, max(1, max(rows)), d
        self.heads = (hq, hk)

    def run(self, causal=True, window=0, out=None, stream=None, workspace=None):
        q = self.q
        out = torch.full_like(q, 3.0) if out is None else out
        lse = torch.full(q.shape[:2], 5.0, dtype=torch.float32, device="cuda")
        status = new_status()
        if workspace is None:
            workspace = torch.zeros(pb.preba_pages_attend_query(len(self.kv), q.shape[0], *self.heads, self.d),
                                    dtype=torch.uint8, device="cuda")
        for _ in range(2):  # the second call finds the workspace as the first left it
            pb.preba_pages_attend(q, self.k, self.v, dev(self.table), dev(self.cu), dev(self.kv), out, workspace,
                                  max_q=self.max_q, scale=self.scale, causal=causal, window=window, lse=lse,
                                  status=status, stream=stream)
        torch.cuda.synchronize()
        return out, host(lse), int(status.item())

    def check(self, causal=True, window=0):
        out, lse, status = self.run(causal, window)
        assert status == 0
        k = torch.nan_to_num(self.k.cpu().double()).numpy()
        v = torch.nan_to_num(self.v.cpu().double()).numpy()
        want, want_lse, spread = ot.attend(host64(self.q), k, v, np.maximum(self.table, 0), self.cu, self.kv,
                                           self.scale, causal, window)
        tol = self.u * np.abs(want) + (self.u + 2.0 ** -14) * spread + 2.0 ** -25 * int(self.kv.max()) * np.abs(v).max()
        got = host64(out)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(),
                               float(np.nanmax(np.abs(got - want))), int(np.isnan(got).sum()))
        assert np.array_equal(np.isinf(lse), np.isinf(want_lse))
        fine = np.isfinite(want_lse)
        assert np.all(np.abs(lse[fine] - want_lse[fine]) <= 2.0 ** -13)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hk,d", [(8, 8, 64), (8, 1, 128), (14, 2, 64), (32, 8, 128), (5, 1, 72), (3, 3, 8),
                                     (16, 1, 120), (40, 8, 96)])
def test_single_tokens(dtype, hq, hk, d):
    Step([(1, 1), (63, 1), (64, 1), (65, 1), (129, 1), (700, 1), (2, 1)], hq, hk, d, 16, dtype).check()


@pytest.mark.parametrize("page,order", [(8, "nhd"), (16, "hnd"), (32, "nhd"), (64, "hnd"), (128, "nhd"),
                                        (256, "hnd")])
def test_pages_and_orders(page, order):
    lengths = [(300, 1), (31, 1), (page, 1), (page + 1, 1)]
    Step(lengths, 8, 2, 128, page, order=order, seed=1).check()
    Step([(300, 40), (31, 31), (page, page), (page + 1, 2)], 8, 2, 64, page, "fp16", order, seed=2).check()


@pytest.mark.parametrize("rows", [2, 3, 4, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257])
def test_chunks_around_the_tiles(rows):
    Step([(rows, rows), (rows + 77, rows), (1, 1)], 4, 1, 64, 16, seed=rows).check()


@pytest.mark.parametrize("hq,hk,d", [(4, 4, 128), (7, 1, 128), (24, 2, 64), (6, 2, 80), (128, 1, 16), (100, 2, 32)])
def test_heads_in_chunks(hq, hk, d):
    Step([(200, 70), (5, 5), (150, 1)], hq, hk, d, 16, "fp16", seed=d).check()


@pytest.mark.parametrize("window", [1, 2, 63, 64, 100, 1000])
@pytest.mark.parametrize("rows", [1, 40])
def test_windows(window, rows):
    kv = [500, 300, 41, 97]
    seen = [max(0, a - rows - window + 1) for a in kv]
    Step([(a, rows) for a in kv], 8, 2, 64, 16, seed=window, first_seen=seen).check(window=window)


@pytest.mark.parametrize("rows", [1, 3, 50])
def test_not_causal(rows):
    Step([(200, rows), (50, rows), (129, rows)], 8, 2, 128, 32, seed=rows).check(causal=False)
    Step([(200, rows), (50, rows), (129, rows)], 8, 2, 128, 32, seed=rows).check(causal=False, window=60)


def test_rows_that_see_nothing():
    # no keys at all, fewer keys than rows, requests without rows
    Step([(0, 1), (0, 3), (1, 1), (5, 0), (0, 0)], 8, 2, 64, 16, seed=1).check()
    Step([(0, 40), (3, 40), (20, 0), (64, 70), (0, 1)], 8, 2, 64, 16, seed=2).check()
    Step([(0, 4), (0, 0)], 8, 2, 128, 16, width=3).check(causal=False)
    Step([(3, 40), (0, 7)], 8, 2, 128, 16, width=3).check(window=2)


def test_long_requests_are_split_and_joined():
    Step([(9000, 1)], 8, 1, 128, 16, seed=1).check()
    Step([(5000, 1), (3, 1), (4097, 1)], 4, 2, 64, 64, "fp16", seed=2).check()
    Step([(6000, 20)], 8, 2, 128, 16, seed=3).check()
    Step([(4000, 3), (900, 40)], 16, 2, 64, 32, "fp16", seed=4).check()


def test_many_requests():
    rng = np.random.default_rng(5)
    Step([(int(a), 1) for a in rng.integers(1, 90, 700)], 4, 2, 64, 16, seed=5).check()
    Step([(int(a) + 9, int(b)) for a, b in zip(rng.integers(1, 90, 150), rng.integers(0, 10, 150))], 4, 1, 64, 16,
         seed=6).check()


def test_large_scores_do_not_overflow():
    for rows in (1, 30):
        s = Step([(300, rows), (40, rows)], 4, 2, 64, 16, "fp16", seed=rows, scale_q=300.0)
        out, lse, status = s.run()
        k, v = (torch.nan_to_num(c.cpu().double()).numpy() for c in (s.k, s.v))
        want, want_lse, spread = ot.attend(host64(s.q), k, v, s.table, s.cu, s.kv, s.scale)
        assert status == 0 and np.isfinite(host64(out)).all() and np.isfinite(lse).all()
        # scores of several hundred: their fp32 sums are off by 2^-22 of sum |q k|, about 2^-9
        assert np.all(np.abs(host64(out) - want) <= s.u * np.abs(want) + (s.u + 2.0 ** -7) * spread + 1e-4)


def test_strided_queries_and_results():
    s = Step([(90, 1), (33, 1)], 8, 2, 64, 16, seed=3)
    c = Step([(90, 20), (33, 9)], 8, 2, 64, 16, seed=3)
    for step in (s, c):
        plain, _, _ = step.run()
        wide = torch.zeros(step.q.shape[0], 11, 72, dtype=step.q.dtype, device="cuda")
        wide[:, 1:9, 8:] = step.q
        step.q, out = wide[:, 1:9, 8:], torch.full((step.q.shape[0], 9, 80), 7.0, dtype=step.q.dtype, device="cuda")
        step.run(out=out[:, :8, 8:72])
        assert torch.equal(out[:, :8, 8:72], plain)
        assert bool((out[:, 8] == 7).all()) and bool((out[:, :, :8] == 7).all()) and bool((out[:, :, 72:] == 7).all())


def test_rows_behind_the_last_request_are_not_written():
    for rows in (1, 30):
        s = Step([(90, rows), (33, rows)], 8, 2, 64, 16, seed=3)
        real = s.q.shape[0]
        s.q = torch.cat([s.q, s.q[:5]])
        out, lse, status = s.run()
        assert status == 0 and bool((out[real:] == 3).all()) and (lse[real:] == 5).all()


def test_results_repeat_bit_for_bit_on_any_stream():
    s = Step([(3000, 1), (77, 1), (1200, 1)], 8, 2, 128, 16, seed=9)
    c = Step([(3000, 50), (77, 7), (1200, 1)], 8, 2, 128, 16, seed=9)
    for step in (s, c):
        first, first_lse, _ = step.run()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            again, again_lse, _ = step.run(stream=side)
            assert torch.equal(first, again) and np.array_equal(first_lse, again_lse)


def test_what_is_out_of_range_is_skipped_and_reported():
    for rows in (1, 30):
        base = dict(hq=8, hk=2, d=64, page=16, seed=4)
        good, _, _ = Step([(90, rows), (40, rows)], **base).run()
        s = Step([(90, rows), (40, rows)], **base)
        s.kv[0] = 16 * s.width + 1
        out, _, status = s.run()
        assert status == pb.ERR_BAD_TABLE and bool((out[:rows] == 3).all()) and torch.equal(out[rows:], good[rows:])
        s = Step([(90, rows), (40, rows)], **base)
        s.kv[1] = -1
        out, _, status = s.run()
        assert status == pb.ERR_BAD_TABLE and bool((out[rows:] == 3).all()) and torch.equal(out[:rows], good[:rows])
        s = Step([(90, rows), (40, rows)], **base)
        s.cu[2] = 2 * rows + 1000
        out, _, status = s.run()
        assert status == pb.ERR_BAD_TABLE and torch.equal(out[:rows], good[:rows])
        for wrong in (-1, 10 ** 6):
            s = Step([(90, rows), (40, rows)], **base)
            s.table[1, 1] = wrong
            out, _, status = s.run()
            assert status == pb.ERR_BAD_TABLE and torch.equal(out[:rows], good[:rows])


def test_a_step_replays_from_a_graph():
    s = Step([(300, 1), (77, 1)], 8, 2, 128, 16, seed=9)
    c = Step([(300, 50), (77, 7)], 8, 2, 128, 16, seed=9)
    for step in (s, c):
        want, _, _ = step.run()
        ws = torch.zeros(pb.preba_pages_attend_query(2, step.q.shape[0], 8, 2, 128), dtype=torch.uint8, device="cuda")
        out, table, cu, kv = torch.zeros_like(step.q), dev(step.table), dev(step.cu), dev(step.kv)
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            pb.preba_pages_attend(step.q, step.k, step.v, table, cu, kv, out, ws, max_q=step.max_q,
                                  scale=step.scale)
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
