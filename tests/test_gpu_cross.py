"""Attention of a decoder's rows to packed states on the GPU against oracle/beams.py.

Tolerances, from the arithmetic.  u is the unit roundoff of the 16-bit type (2^-8 bfloat16, 2^-11 binary16): one rounding
of the result, one of each probability (u sum p|v| / sum p), scores whose fp32 sums are off by at most 2^-15 (twice,
for numerator and denominator: 2^-14), and probabilities below the type's normal range, off by 2^-25 of the
reference each: u |out| + (u + 2^-14) spread + 2^-25 states max|v|.  The log-sum-exp is off by no more than the scores
and a few fp32 roundings: 2^-13.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import beams as ob
from paper_2411_19114_b200 import binding as pb

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}


def ints(a):
    return torch.as_tensor(np.ascontiguousarray(a)).to(torch.int32).cuda()


def host64(t):
    return t.cpu().double().numpy()


def starts(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(int)


class Step:
    """A call's operands in the forms that a program has them: queries of one projection, keys and values of another, each
    with room around them; results between guards."""

    def __init__(self, rows, states, hq, hk, d, dtype, seed=0, spread=2.0, seen=None, slack=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dt, self.u = DTYPES[dtype]
        self.cu_q, self.cu_k = starts(rows), starts(states)
        tokens, total = int(self.cu_q[-1]), int(self.cu_k[-1])
        self.tokens, self.max_q, self.scale = tokens, max(1, max(rows)), d ** -0.5
        qs = torch.randn(tokens + slack, hq + 1, d, generator=g, device="cuda").mul_(spread).to(self.dt)
        kv = torch.randn(total + slack, 2, hk, d, generator=g, device="cuda").to(self.dt)
        kv[total:] = float("nan")  # behind the last state
        self.q, self.k, self.v = qs[:tokens, :hq], kv[:, 0], kv[:, 1]
        self.seen = seen
        self.whole = torch.full((tokens + slack, hq, d + 8), 7.0, dtype=self.dt, device="cuda")
        self.lse = torch.full((tokens, hq), 7.0, device="cuda")
        self.status = ints([0])
        need = pb.preba_cross_attend_query(len(rows), max(1, tokens), hq, hk, d)
        self.ws = torch.zeros(need + 64, dtype=torch.uint8, device="cuda")
        self.ws[need:] = 0x5a
        self.need, self.d, self.slack = need, d, slack

    def call(self, **kwargs):
        args = dict(max_q=self.max_q, scale=self.scale, seen=None if self.seen is None else ints(self.seen), lse=self.lse,
                    status=self.status)
        args.update(kwargs)
        pb.preba_cross_attend(self.q, self.k, self.v, ints(self.cu_q), ints(self.cu_k), self.whole[:self.tokens, :, :self.d],
                              self.ws[:self.need], **args)

    def out(self):
        torch.cuda.synchronize()
        assert bool((self.whole[self.tokens:] == 7).all()) and bool((self.whole[..., self.d:] == 7).all())
        assert bool((self.ws[self.need:] == 0x5a).all()) and not bool(self.ws[:640].any())
        return self.whole[:self.tokens, :, :self.d]

    def check(self):
        self.call()
        got = self.out().clone()
        lse = self.lse.clone()
        assert int(self.status.item()) == 0
        self.call()  # the same call gives the same bits
        assert torch.equal(self.out().view(torch.int16), got.view(torch.int16)) and torch.equal(self.lse, lse)
        want, want_lse, spread = ob.cross_attend(host64(self.q), host64(self.k), host64(self.v), self.cu_q, self.cu_k, self.scale,
                                                 self.seen)
        states = int(np.diff(self.cu_k).max())
        tol = self.u * np.abs(want) + (self.u + 2.0 ** -14) * spread + 2.0 ** -25 * states * float(
            np.abs(np.nan_to_num(host64(self.v))).max())
        assert np.all(np.abs(host64(got) - want) <= tol)
        empty = np.isinf(want_lse)
        assert np.array_equal(np.isinf(lse.cpu().numpy()), empty)
        assert np.all(np.abs(host64(lse)[~empty] - want_lse[~empty]) <= 2.0 ** -13)
        assert not host64(got)[empty].any()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,states,hq,hk,d", [
    ([1], [1], 1, 1, 8), ([1], [128], 2, 1, 64), ([1], [129], 1, 1, 128), ([4, 4], [375, 90], 8, 8, 64),
    ([5] * 7, [1, 2, 127, 128, 129, 700, 31], 3, 3, 64), ([8] * 3, [300, 1, 640], 8, 2, 128), ([16], [513], 4, 1, 80),
    ([3, 0, 2, 3], [40, 50, 0, 256], 6, 2, 72), ([0, 0, 1], [9, 0, 3], 2, 2, 64), ([64], [5000], 1, 1, 64),
    ([2], [20000], 7, 1, 128), ([4] * 40, list(range(1, 161, 4)), 4, 4, 40), ([1] * 300, [7] * 300, 2, 1, 64),
    ([1], [3], 64, 1, 64), ([13], [300], 5, 1, 128),
    # as many rows as the kernel takes, and one more
    ([32, 5], [300, 1], 3, 3, 64), ([33, 5], [300, 1], 3, 3, 64), ([64], [300], 2, 2, 128), ([65], [300], 2, 2, 128),
    # runs that end with a piece's beginning but no tile of it
    ([16, 2], [30000, 500], 2, 1, 128), ([2] * 5, [20000, 128 * 89, 128 * 90, 128 * 91, 40000], 3, 1, 64)])
def test_few_rows_match_the_definition(rows, states, hq, hk, d, dtype):
    Step(rows, states, hq, hk, d, dtype, seed=len(rows) + d).check()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,states,hq,hk,d", [
    ([65], [1], 1, 1, 64), ([200], [333], 2, 2, 64), ([1], [90], 65, 1, 128), ([130, 1, 77, 0], [129, 500, 0, 20], 4, 2, 80),
    ([40] * 6, [257, 1, 128, 60, 300, 2], 6, 3, 64), ([300], [3000], 1, 1, 128), ([30] * 70, [20] * 70, 6, 1, 64),
    ([700, 3], [5, 600], 2, 2, 128)])
def test_many_rows_match_the_definition(rows, states, hq, hk, d, dtype):
    Step(rows, states, hq, hk, d, dtype, seed=len(rows) + d).check()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,states,hq,hk,d", [
    ([4, 7, 2], [600, 90, 300], 4, 2, 64), ([30], [900], 2, 1, 128), ([90, 200, 70], [400, 130, 1000], 4, 2, 64),
    ([300], [700], 1, 1, 128)])
def test_rows_see_the_first_states_only(rows, states, hq, hk, d, dtype):
    rng = np.random.default_rng(sum(rows))
    most = np.repeat(states, rows)
    for kind in range(4):
        seen = rng.integers(-2, most + 3)  # in no order; more than there are, and fewer than none
        if kind == 1:
            seen = np.sort(seen)
        elif kind == 2:
            seen[:] = 0
            seen[len(seen) // 2] = most[len(seen) // 2]  # one row sees all, the others nothing
        elif kind == 3:
            seen = np.minimum(seen, 3)
        Step(rows, states, hq, hk, d, dtype, seed=kind, seen=seen).check()


@pytest.mark.parametrize("rows", [[3, 2], [150, 90]])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_states_that_no_row_sees_may_hold_anything(rows, dtype):
    for bad in (float("nan"), float("inf"), -float("inf")):
        s = Step(rows, [300, 77], 4, 2, 64, dtype, seed=3, seen=np.repeat([170, 50], rows))
        s.check()
        want = s.out().clone()
        for first, last in ((170, 300), (350, 377)):
            s.k[first:last], s.v[first:last] = bad, bad
        s.call()
        assert torch.equal(s.out(), want)


@pytest.mark.parametrize("rows", [[5], [70]])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_scores_that_grow_fall_and_are_far_apart(rows, dtype):
    for kind in range(3):
        s = Step(rows, [1500], 2, 1, 64, dtype, seed=kind)
        ramp = torch.linspace(0, 6, 1500, device="cuda")[:, None, None]
        if kind == 0:
            s.k[:1500].mul_(ramp)  # references grow tile by tile
        elif kind == 1:
            s.k[:1500].mul_(6 - ramp)
        else:
            s.k[700].mul_(20)  # one state outdoes all
        # scores up to 20 * 2^4: their sums are off by as much more
        got = (s.call(), s.out().clone())[1]
        want, _, spread = ob.cross_attend(host64(s.q), host64(s.k), host64(s.v), s.cu_q, s.cu_k, s.scale)
        far = 2.0 ** -18 * 64 * float(s.k[:1500].abs().max()) * float(s.q.abs().max()) * s.scale
        assert np.all(np.abs(host64(got) - want) <= s.u * np.abs(want) + (s.u + 2.0 ** -14 + far) * spread + 2.0 ** -25 * 1500 * 6)


@pytest.mark.parametrize("rows", [[3], [70]])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_scores_that_are_not_numbers_and_scores_of_minus_infinity(rows, dtype):
    s = Step(rows, [500], 1, 1, 64, dtype)
    s.q[1, 0, 0] = float("nan")
    s.call()
    got = s.out().float()
    assert bool(got[1].isnan().all()) and bool(s.lse[1].isnan().all())
    assert not bool(got[0].isnan().any()) and not bool(got[2].isnan().any())
    s = Step(rows, [500], 1, 1, 64, dtype)
    s.q[:, :, 0], s.k[:, :, 0] = 1, -float("inf")  # every score is -inf
    s.call()
    assert not bool(s.out().any()) and bool((s.lse == -float("inf")).all())
    s = Step(rows, [500], 1, 1, 64, dtype)
    s.q[:, :, 0], s.k[:, :, 0] = 1, 0
    s.k[:400, :, 0] = -float("inf")  # of the first tiles only
    s.call()
    want, _, _ = ob.cross_attend(host64(s.q), host64(s.k[400:]), host64(s.v[400:]), s.cu_q, [0, 100], s.scale)
    assert np.all(np.abs(host64(s.out()) - want) <= 4 * s.u * 4)


@pytest.mark.parametrize("rows", [[3, 2, 4], [90, 2, 70]])
def test_requests_at_fault_are_skipped(rows):
    for cu_q, cu_k, max_q in (([0, 0, 2, 1], None, None), (None, [0, 300, 200, 500], None), (None, [0, 100, 200, 10 ** 6], None),
                              (None, [-5, 100, 200, 300], None), (None, None, max(rows) - 1)):
        s = Step(rows, [100, 100, 100], 2, 2, 64, "bf16")
        good_q, good_k = s.cu_q, s.cu_k
        if cu_q is not None:
            s.cu_q = np.array([good_q[0], good_q[1], good_q[-1] + 5, good_q[2]])
        if cu_k is not None:
            s.cu_k = np.array(cu_k)
        s.call(max_q=max_q or s.max_q)
        got = s.out()
        assert int(s.status.item()) == pb.ERR_BAD_TABLE
        for r in range(3):
            a, b, c, e = s.cu_q[r], s.cu_q[r + 1], s.cu_k[r], s.cu_k[r + 1]
            ok = 0 <= a <= b <= s.tokens and b - a <= (max_q or s.max_q) and 0 <= c <= e <= 303
            if not ok and 0 <= a <= b <= s.tokens:
                assert bool((got[a:b] == 7).all())
            if ok:
                want, _, spread = ob.cross_attend(host64(s.q[a:b]), host64(s.k[c:e]), host64(s.v[c:e]), [0, b - a], [0, e - c], s.scale)
                assert np.all(np.abs(host64(got[a:b]) - want) <= s.u * np.abs(want) + (s.u + 2.0 ** -14) * spread + 2.0 ** -25 * 600)


def test_requests_whose_states_overlap_are_no_longer_a_line_and_do_no_harm():
    """Every other request has all the states: far more tiles than any packed call."""
    n, states, hk = 16384, 1 << 22, 128
    s = Step([1] * n, [1] * n, hk, hk, 8, "fp16", slack=0)
    s.k = s.v = torch.zeros((states + hk) * 8, dtype=torch.float16, device="cuda").as_strided((states, hk, 8), (8, 8, 1))
    s.cu_k = np.tile([0, states], n // 2 + 1)[:n + 1]
    s.call()
    s.out()
    assert int(s.status.item()) == pb.ERR_BAD_TABLE


@pytest.mark.parametrize("rows", [[4] * 5, [100, 60]])
def test_captured_calls_replay_on_new_inputs(rows):
    s = Step(rows, [300] * len(rows), 4, 2, 64, "bf16")
    cu_q, cu_k = ints(s.cu_q), ints(s.cu_k)
    out, ws = s.whole[:s.tokens, :, :s.d], s.ws[:s.need]
    call = pb.PreparedCrossAttend(s.q, s.k, s.v, cu_q, cu_k, out, ws, max_q=s.max_q, scale=s.scale, status=s.status)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        call()
    for shorter in (300, 200, 1):
        s.cu_k = starts([shorter] * len(rows))
        cu_k.copy_(ints(s.cu_k))
        s.q.normal_()
        s.whole.fill_(7)
        graph.replay()
        got = s.out().clone()
        s.whole.fill_(7)
        call()
        assert torch.equal(s.out(), got)
        want, _, spread = ob.cross_attend(host64(s.q), host64(s.k), host64(s.v), s.cu_q, s.cu_k, s.scale)
        assert np.all(np.abs(host64(got) - want) <= s.u * np.abs(want) + (s.u + 2.0 ** -14) * spread + 2.0 ** -25 * 300 * 6)


def test_a_step_without_rows_and_calls_on_two_streams():
    a, b = Step([5] * 9, [700] * 9, 8, 8, 64, "bf16", seed=1), Step([130] * 3, [700] * 3, 8, 8, 64, "bf16", seed=2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    want = []
    for s in (a, b):
        s.call()
        want.append(s.out().clone())
        s.whole.fill_(7)
    torch.cuda.synchronize()
    calls = [pb.PreparedCrossAttend(s.q, s.k, s.v, ints(s.cu_q), ints(s.cu_k), s.whole[:s.tokens, :, :s.d], s.ws[:s.need],
                                    max_q=s.max_q, scale=s.scale, stream=st) for s, st in zip((a, b), streams)]
    torch.cuda.synchronize()
    for _ in range(20):
        for c in calls:
            c()
    for s, w in zip((a, b), want):
        assert torch.equal(s.out(), w)


@pytest.mark.parametrize("rows,states,hq,hk,d", [([90, 200, 70], [400, 130, 1000], 4, 2, 64), ([60, 33], [400, 900], 4, 4, 64),
                                                 ([12, 9, 16], [800, 500, 300], 4, 2, 64)])
def test_rows_of_very_different_limits_give_the_same_bits_every_time(rows, states, hq, hk, d):
    """Warps whose rows see little, or are not there, are done with a tile before the others."""
    rng = np.random.default_rng(sum(rows))
    most = np.repeat(states, rows)
    for seed in range(40):
        s = Step(rows, states, hq, hk, d, "bf16", seed=seed, seen=rng.integers(-2, most + 3))
        s.call()
        want = s.out().clone()
        for _ in range(3):
            s.whole.fill_(7)
            s.call()
            assert torch.equal(s.out(), want), seed
        if seed == 0:
            s.check()
