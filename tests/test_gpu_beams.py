"""Beam selection, block tables of the beams and copies of their open pages on the GPU against
oracle/beams.py.

Tolerance of the selection's values, from the arithmetic: an exponential is off by 2^-22 of itself (ex2.approx) and by
its argument's error, 2^-22.5 |x - max|, which weighs |x - max| e^-|x - max| < 0.37; a segment's sum of positive terms has
at most 37 roundings one after the other, 37 * 2^-24 < 2^-18.7.  The sum of segments is 64-bit.  So
the logarithm is off by less than 2^-18, and the value is rounded once: 2^-24 of itself.  Order within a row does not
depend on any of this.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import beams as ob
from paper_2411_19114_b200 import binding as pb

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
INF = float("inf")


def ints(a):
    return torch.as_tensor(np.ascontiguousarray(a)).to(torch.int32).cuda()


def run_select(logits, scores, width, beams, end=-1, done=None, allowed=None, weights=None):
    """``logits`` a CUDA tensor, the rest numpy; every output is laid out between guards."""
    rows, vocab = logits.shape
    n = rows // beams
    out = [torch.full((n + 2, width), -7, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    flags = torch.full((n + 2, width), 7, dtype=torch.uint8, device="cuda")
    bits = None
    if allowed is not None:
        words = np.zeros((len(allowed), -(-vocab // 32) * 32), dtype=np.uint8)
        words[:, :vocab] = allowed
        bits = torch.from_numpy(np.packbits(words, axis=1, bitorder="little").view(np.int32).copy()).cuda()
    status = ints([0])
    size = pb.preba_beam_select_query(n, beams, width, vocab, logits.dtype)
    f32 = lambda a: None if a is None else torch.tensor(np.asarray(a, dtype=np.float32)).cuda()  # noqa: E731
    ws = torch.full((size + 64,), 0xff, dtype=torch.uint8, device="cuda")  # whatever it holds
    got = [t[1:n + 1] for t in out]
    for _ in range(2):
        pb.preba_beam_select(logits, f32(scores), *got, ws[:size], end_token=end,
                             done=None if done is None else torch.tensor(done).to(torch.uint8).cuda(), done_out=flags[1:n + 1],
                             allowed=bits, weights=f32(weights), status=status)
    torch.cuda.synchronize()
    for t in (*out, flags):
        assert bool((t[0] == t[n + 1]).all()) and float(t[0, 0]) in (-7, 7)
    assert bool((ws[size:] == 0xff).all())
    return (*(t.cpu().numpy() for t in got), flags[1:n + 1].cpu().numpy(), int(status.item()))


def check_select(got, want):
    tokens, parents, scores, done, bad = want
    assert np.array_equal(got[0], tokens)
    assert np.array_equal(got[1], parents)
    assert np.array_equal(got[3], done.astype(np.uint8))
    assert np.array_equal(np.isinf(got[2]), np.isinf(scores))
    seen = np.isfinite(scores)
    assert np.all(np.abs(got[2][seen] - scores[seen]) <= 2.0 ** -18 + 2.0 ** -24 * np.abs(scores[seen]))
    assert got[4] == (pb.ERR_BAD_TABLE if bad else 0)


def made(rng, rows, vocab, dtype, coarse=False):
    x = rng.normal(size=(rows, vocab)) * 2
    x[np.arange(rows)[:, None], rng.integers(0, vocab, (rows, 6))] += 8 * rng.random((rows, 6))
    if coarse:
        x = np.round(x)  # a row's best are many times the same
    t = torch.tensor(x).to(DTYPES[dtype])
    return t.cuda(), t.double().numpy()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("n,beams,width,vocab", [
    (1, 1, 1, 1), (1, 1, 64, 3), (2, 3, 4, 31), (3, 4, 4, 1000), (2, 5, 10, 1024), (2, 8, 8, 2048), (1, 32, 64, 1025),
    (5, 4, 8, 5003), (33, 2, 3, 4097), (1, 6, 6, 50001), (2, 32, 32, 512), (4, 17, 5, 2049)])
def test_selection_matches_the_definition(n, beams, width, vocab, dtype):
    rng = np.random.default_rng(n * 1000 + vocab)
    x, x64 = made(rng, n * beams, vocab, dtype)
    scores = (-rng.random(n * beams) * 6).astype(np.float32)
    check_select(run_select(x, scores, width, beams), ob.select(x64, scores, width, beams))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("vocab,pad", [(777, 0), (2560, 0), (4099, 5), (9000, 8)])
def test_selection_with_masks_ended_beams_weights_and_many_equals(vocab, pad, dtype):
    n, beams, width = 4, 5, 12
    rng = np.random.default_rng(vocab)
    x, x64 = made(rng, n * beams, vocab + pad, dtype, coarse=True)
    x, x64 = x[:, pad:], x64[:, pad:]  # rows with a stride, that begin anywhere
    scores = (-rng.random(n * beams) * 4).astype(np.float32)
    done = rng.random(n * beams) < 0.3
    done[:beams] = True  # a request whose beams have all ended has no more candidates than beams
    weights = rng.uniform(0.2, 1.5, n * beams).astype(np.float32)
    allowed = rng.random((n * beams, vocab)) < 0.1
    allowed[7] = False  # nothing is left of this row
    for mask in (allowed, allowed[:1]):
        check_select(run_select(x, scores, width, beams, 5, done, mask, weights),
                     ob.select(x64, scores, width, beams, 5, done, mask, weights))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_equal_values_go_to_the_lowest_beam_and_token(dtype):
    vocab, beams, width = 3001, 4, 9  # odd: rows begin at different places of a vector
    for x64 in (np.zeros((beams, vocab)), np.tile(np.round(np.random.default_rng(1).normal(size=vocab)), (beams, 1))):
        x = torch.tensor(x64).to(DTYPES[dtype]).cuda()
        tokens, parents, *_ = run_select(x, np.full(beams, -1.5), width, beams)
        top = np.flatnonzero(x64[0] == x64[0].max())[:width]
        flat = [(b, t) for b in range(beams) for t in top][:width] if len(top) < width else [(0, t) for t in top]
        if len(top) * beams >= width:
            assert list(zip(parents[0], tokens[0])) == flat
        check_select(run_select(x, np.full(beams, -1.5), width, beams), ob.select(x64, np.full(beams, -1.5), width, beams))
    x = torch.tensor([[0.0, -0.0, 0.0, -0.0]]).to(DTYPES[dtype]).cuda()
    assert run_select(x, [0.0], 4, 1)[0].tolist() == [[0, 1, 2, 3]]


def test_logits_at_odd_addresses_and_of_a_wider_buffer():
    rng = np.random.default_rng(5)
    for dtype in ("bf16", "fp16", "fp32"):
        for shift in range(1, 9):
            whole, whole64 = made(rng, 6, 2200, dtype)
            x, x64 = whole[:, shift:2101 + shift], whole64[:, shift:2101 + shift]
            scores = (-rng.random(6)).astype(np.float32)
            check_select(run_select(x, scores, 5, 3), ob.select(x64, scores, 5, 3))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_that_offer_nothing_and_rows_at_fault(dtype):
    rng = np.random.default_rng(9)
    vocab, beams = 1500, 3
    for fault in range(9):
        x, x64 = made(rng, 2 * beams, vocab, dtype)
        scores, weights, done, allowed = -rng.random(6).astype(np.float32), np.ones(6, np.float32), np.zeros(6, bool), np.ones((6, vocab), bool)
        if fault == 0:
            x[1, 1400] = float("nan")
        elif fault == 1:
            x[1, 3] = INF
        elif fault == 2:
            x[1] = -INF
        elif fault == 3:
            x[1], allowed[1] = float("nan"), False
        elif fault == 4:
            x[1], scores[1] = float("nan"), -INF
        elif fault == 5:
            x[1], done[1] = float("nan"), True
        elif fault == 6:
            scores[1] = float("nan")
        elif fault == 7:
            weights[1] = -1
        else:  # not a number beside -inf only
            x[1] = -INF
            x[1, 700] = float("nan")
        x64 = x.double().cpu().numpy()
        check_select(run_select(x, scores, 6, beams, 2, done, allowed, weights),
                     ob.select(x64, scores, 6, beams, 2, done, allowed, weights))
    # the first step: one beam is there
    x, x64 = made(rng, 4, vocab, dtype)
    scores = np.array([0, -INF, -INF, -INF], dtype=np.float32)
    got = run_select(x, scores, 4, 4)
    check_select(got, ob.select(x64, scores, 4, 4))
    assert (got[1] == 0).all()


def test_selection_of_far_values():
    """Scores of long hypotheses, logits that are far apart and near the end of their type's range."""
    rng = np.random.default_rng(3)
    x, _ = made(rng, 8, 3000, "bf16")
    x.mul_(1e36)
    scores = (-rng.random(8) * 1e4).astype(np.float32)
    got, want = run_select(x, scores, 4, 4), ob.select(x.double().cpu().numpy(), scores, 4, 4)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    assert np.all(np.abs(got[2] - want[2]) <= 2.0 ** -18 + 2.0 ** -22 * np.abs(want[2]))


# ---- block tables ---------------------------------------------------------------------------------

def beam_state(rng, n, beams, page, longest, spread=True):
    """Rows that share pages from the left, each with a last page of its own."""
    lengths = rng.integers(0, longest + 1, n * beams) if spread else np.repeat(rng.integers(0, longest + 1, n), beams)
    held = -(-lengths // page)
    width = max(1, int(held.max()) + 1)
    table, number = np.full((n * beams, width), -1), 0
    for i in range(n * beams):
        share = 0
        if i % beams:
            share = int(rng.integers(0, min(lengths[i - 1], lengths[i]) // page + 1))
        table[i, :share] = table[i - 1, :share]
        table[i, share:held[i]] = number + np.arange(held[i] - share)
        number += held[i] - share
    order = rng.permutation(number + n * beams + 5)
    table = np.where(table >= 0, order[table], -1)
    return lengths, table, order[number:], len(order)


def run_pages(parents, lengths, table, beams, page, free, count, capacity, total, kept=None):
    rows, width = table.shape
    n = rows // beams
    stack = ints(np.concatenate([free, np.full(max(0, capacity - len(free)), -9)])[:capacity]) if capacity else ints([0])
    out = torch.full((rows + 2, width + 3), -7, dtype=torch.int32, device="cuda")  # rows with a stride, between guards
    lengths_out, copies = ints(np.full(rows, -7)), torch.full((rows, 4), -7, dtype=torch.int32, device="cuda")
    left, status = ints([-7]), ints([0])
    size = pb.preba_beam_pages_query(n, beams, width)
    ws = torch.full((size + 64,), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(2):  # twice: the call changes nothing that it reads
        pb.preba_beam_pages(ints(parents), ints(lengths), ints(table), out[1:-1, :width], lengths_out, copies, stack, ints([count]),
                            left, page, ws[:size], beams, pages=total, kept=None if kept is None else ints(kept), status=status)
    torch.cuda.synchronize()
    assert bool((out[0] == -7).all()) and bool((out[-1] == -7).all()) and bool((out[:, width:] == -7).all())
    assert bool((ws[size:] == 0xff).all())
    return dict(table=out[1:-1, :width].cpu().numpy(), lengths=lengths_out.cpu().numpy(), copies=copies.cpu().numpy(),
                free=stack.cpu().numpy(), left=int(left.item()), status=int(status.item()))


def check_pages(got, want, either=False):
    for name in ("table", "lengths", "copies", "free"):
        assert np.array_equal(got[name], want[name]), name
    assert got["left"] == want["left"]
    faults = [pb.ERR_BAD_TABLE] * want["bad"] + [pb.ERR_BUFFER_TOO_SMALL] * want["short"]
    assert got["status"] in faults if faults else got["status"] == 0


def both(parents, lengths, table, beams, page, free, count, capacity, total, kept=None):
    memory = np.concatenate([free, np.full(max(0, capacity - len(free)), -9)])[:capacity]
    got = run_pages(parents, lengths, table, beams, page, free, count, capacity, total, kept)
    want = ob.pages(parents, lengths, table, beams, page, memory, count, capacity, total, kept)
    check_pages(got, want)
    return got, want


@pytest.mark.parametrize("n,beams,page,longest,spread", [
    (1, 1, 16, 40, False), (1, 4, 16, 600, False), (3, 8, 8, 300, True), (2, 32, 16, 200, True), (5, 5, 32, 9000, False),
    (1, 3, 8, 5000, True), (700, 4, 16, 60, False), (1100, 3, 16, 30, True), (512, 32, 64, 100, False), (2, 2, 256, 0, True),
    (16384, 1, 16, 40, True), (5461, 3, 32, 40, False), (3, 9, 8, 2100, True)])
def test_tables_match_the_definition(n, beams, page, longest, spread):
    rng = np.random.default_rng(n + beams)
    lengths, table, free, total = beam_state(rng, n, beams, page, longest, spread)
    for low in (0, -1):  # with and without rows that end
        parents = np.minimum((rng.random(n * beams) ** 2 * (beams - low)).astype(int) + low, beams - 1)
        both(parents, lengths, table, beams, page, free, len(free), total, total)
    kept = rng.integers(0, 3, n)
    both(parents, lengths, table, beams, page, free, len(free), total, total, kept)


def test_beams_that_stay_change_nothing_and_a_beam_that_takes_all_shares_its_pages():
    rng = np.random.default_rng(2)
    lengths, table, free, total = beam_state(rng, 3, 4, 16, 100, False)
    same = np.tile(np.arange(4), 3)
    got, _ = both(same, lengths, table, 4, 16, free, len(free), total, total)
    held = -(-lengths // 16)
    assert all(np.array_equal(got["table"][i, :held[i]], table[i, :held[i]]) for i in range(12))
    assert got["left"] == len(free) and not got["copies"].any()
    got, _ = both(np.full(12, 2), lengths, table, 4, 16, free, len(free), total, total)
    full = lengths[2] // 16
    assert all(np.array_equal(got["table"][i, :full], table[2, :full]) for i in range(4))
    assert len({int(got["table"][i, full]) for i in range(4)}) == (4 if lengths[2] % 16 else 1) or lengths[2] % 16 == 0


@pytest.mark.parametrize("count", [0, 1, 2, 3, 5, 8, 13])
def test_requests_that_the_pages_do_not_suffice_for_are_refused_in_order(count):
    rng = np.random.default_rng(count)
    for beams, n in ((4, 9), (3, 1200)):
        lengths, table, free, total = beam_state(rng, n, beams, 16, 70, False)
        parents = (rng.random(n * beams) ** 3 * beams).astype(int)
        both(parents, lengths, table, beams, 16, free, count, total, total)


def test_tables_at_fault():
    rng = np.random.default_rng(4)
    lengths, table, free, total = beam_state(rng, 6, 4, 16, 100, False)
    parents = rng.integers(0, 4, 24)
    bad = lengths.copy()
    bad[5], bad[9] = -3, 16 * table.shape[1] + 1  # longer than the row of the table
    both(parents, bad, table, 4, 16, free, len(free), total, total)
    wrong = parents.copy()
    wrong[7] = 4
    both(wrong, lengths, table, 4, 16, free, len(free), total, total)
    broken = table.copy()
    broken[rng.random(table.shape) < 0.3] = total + 3
    both(np.full(24, 1), lengths, broken, 4, 16, free, len(free), total, total)
    # a stack with unusable pages, one without room, and a count that is out of range
    both(parents, lengths, table, 4, 16, np.full_like(free, total), len(free), total, total)
    both(np.full(24, -1), lengths, table, 4, 16, free, len(free), len(free) + 2, total)
    for count in (-1, total + 1):
        got = run_pages(np.tile(np.arange(4), 6), lengths, table, 4, 16, free, count, total, total)
        assert got["status"] == pb.ERR_BAD_TABLE and got["left"] == 0


# ---- copies ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rows,layers,page,hk,d,order", [
    (1, 1, 8, 1, 8, "nhd"), (7, 3, 16, 2, 64, "nhd"), (40, 2, 32, 5, 80, "hnd"), (3, 128, 16, 1, 128, "hnd"),
    (2100, 1, 16, 1, 16, "nhd"), (9, 2, 256, 3, 72, "nhd")])
def test_copies_move_the_slots_they_name_and_nothing_else(rows, layers, page, hk, d, order, dtype):
    rng = np.random.default_rng(rows + d)
    total = 2 * rows + 6
    numbers = rng.permutation(total)
    copies = np.stack([numbers[:rows], numbers[rows:2 * rows], rng.integers(0, page + 1, rows), np.zeros(rows)], 1).astype(int)
    copies[rows // 2, 0] = copies[0, 0]  # two copies of one page
    g = torch.Generator(device="cuda").manual_seed(rows)
    shape = (total, page, hk, d) if order == "nhd" else (total, hk, page, d)
    made = [torch.randn((total, *shape[1:3], d + 8), generator=g, device="cuda").to(DTYPES[dtype])[..., :d] for _ in range(2 * layers)]
    caches = made if order == "nhd" else [c.transpose(1, 2) for c in made]
    want = [c.clone() for c in caches]
    for w in want:
        for source, to, count, _ in copies:
            w[to, :count] = w[source, :count]
    status = ints([0])
    for _ in range(2):
        pb.preba_pages_copy(ints(copies), caches[:layers], caches[layers:], status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert all(torch.equal(c.view(torch.int16) if c.is_contiguous() else c, w.view(torch.int16) if c.is_contiguous() else w)
               for c, w in zip(caches, want))


def test_copies_at_fault_are_left_out():
    c = torch.arange(4 * 8 * 8, device="cuda").half().view(4, 8, 1, 8)
    for entry in ([-1, 1, 3, 0], [4, 1, 3, 0], [0, 4, 3, 0], [0, -1, 3, 0], [0, 1, 9, 0], [0, 1, -2, 0]):
        k, v, status = c.clone(), c.clone(), ints([0])
        pb.preba_pages_copy(ints([[2, 3, 8, 0], entry]), [k], [v], status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == pb.ERR_BAD_TABLE
        want = c.clone()
        want[3] = want[2]
        assert torch.equal(k, want) and torch.equal(v, want)


@pytest.mark.parametrize("dtype,vocab,masked", [("bf16", 140001, False), ("fp16", 140000, True), ("fp32", 70003, True)])
def test_selection_where_every_warp_has_many_segments(dtype, vocab, masked):
    """More segments than the GPU has warps, several times over; rows of all kinds among them."""
    n, beams, width = 32, 8, 8
    rng = np.random.default_rng(vocab)
    x, x64 = made(rng, n * beams, vocab, dtype)
    scores = (-rng.random(n * beams) * 6).astype(np.float32)
    scores[rng.random(n * beams) < 0.1] = -INF
    done = rng.random(n * beams) < 0.2
    allowed = rng.random((1, vocab)) < 0.5 if masked else None
    check_select(run_select(x, scores, width, beams, 7, done, allowed), ob.select(x64, scores, width, beams, 7, done, allowed))


@pytest.mark.parametrize("width", [1, 3, 20, 64])
def test_equal_logits_in_many_segments(width):
    """More segments of the same maximum than a request may list."""
    vocab, beams = 180001, 3
    x = torch.full((2 * beams, vocab), 1.25, dtype=torch.float16, device="cuda")
    scores = np.array([-1, -1, -2, -3, -3, -3], dtype=np.float32)
    done = np.array([False, True, False, True, True, True])
    for ended in (None, done):
        got = run_select(x, scores, width, beams, 9 if ended is not None else -1, ended)
        check_select(got, ob.select(x.double().cpu().numpy(), scores, width, beams, 9 if ended is not None else -1, ended))


@pytest.mark.parametrize("weights", [[1e-40, 1e-40, 2e-40], [1e-44, 1.0, 1e-44], [3e38, 1e38, 2e38]])
@pytest.mark.parametrize("score", [300.0, -300.0])
def test_weights_whose_reciprocals_leave_the_type(weights, score):
    beams, width = 3, 5
    rng = np.random.default_rng(4)
    logits, x = made(rng, 2 * beams, 5000, "fp32")
    scores = np.float32(score + 10 * rng.random(2 * beams))
    w = np.float32(weights * 2)
    check_select(run_select(logits, scores, width, beams, weights=w), ob.select(x, scores, width, beams, weights=w))
