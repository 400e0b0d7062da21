"""Selection, tables and copies captured in a graph and replayed on other inputs, and made again under another stream."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import beams as ob
from paper_2411_19114_b200 import binding as pb
from test_gpu_beams import beam_state, check_pages, ints, made

pytestmark = pytest.mark.gpu


class Calls:
    """A step's three calls on buffers that stay."""

    def __init__(self, n=6, beams=4, vocab=3001, page=16, layers=3, seed=0):
        self.n, self.beams, self.vocab, self.page = n, beams, vocab, page
        self.rng = np.random.default_rng(seed)
        rows = n * beams
        self.logits, _ = made(self.rng, rows, vocab, "bf16")
        self.scores = torch.zeros(rows, device="cuda")
        self.tokens, self.parents = ints(np.zeros((n, beams))), ints(np.zeros((n, beams)))
        self.values, self.status = torch.zeros(n, beams, device="cuda"), ints([0])
        self.lengths64, self.table64, self.free64, self.total = beam_state(self.rng, n, beams, page, 200, False)
        self.lengths, self.table = ints(self.lengths64), ints(self.table64)
        self.table_out, self.lengths_out = torch.full_like(self.table, -7), torch.zeros_like(self.lengths)
        self.copies, self.count, self.left = ints(np.zeros((rows, 4))), ints([len(self.free64)]), ints([0])
        self.memory = np.concatenate([self.free64, np.full(self.total - len(self.free64), -9)])
        self.free = ints(self.memory)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.caches = [torch.randn(self.total, page, 2, 64, generator=g, device="cuda").half() for _ in range(2 * layers)]
        ws = lambda size: torch.zeros(size, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.calls = [
            pb.PreparedBeamSelect(self.logits, self.scores, self.tokens, self.parents, self.values,
                                  ws(pb.preba_beam_select_query(n, beams, beams, vocab, torch.bfloat16)), status=self.status),
            pb.PreparedBeamPages(self.parents, self.lengths, self.table, self.table_out, self.lengths_out, self.copies, self.free,
                                 self.count, self.left, page, ws(pb.preba_beam_pages_query(n, beams, self.table.shape[1])), beams,
                                 pages=self.total, status=self.status),
            pb.PreparedPagesCopy(self.copies, self.caches[:layers], self.caches[layers:], status=self.status)]

    def __call__(self):
        for c in self.calls:
            c()

    def renew(self):
        fresh, _ = made(self.rng, self.n * self.beams, self.vocab, "bf16")
        self.logits.copy_(fresh)
        self.scores.copy_(torch.tensor(-self.rng.random(self.n * self.beams) * 5))
        self.free.copy_(ints(self.memory))
        self.table_out.fill_(-7)
        self.before = [c.clone() for c in self.caches]

    def check(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        host = lambda t: t.cpu().numpy()  # noqa: E731
        tokens, parents, *_ = ob.select(self.logits.double().cpu().numpy(), host(self.scores), self.beams, self.beams)
        assert np.array_equal(host(self.tokens), tokens) and np.array_equal(host(self.parents), parents)
        want = ob.pages(parents.flatten(), self.lengths64, self.table64, self.beams, self.page, self.memory, len(self.free64),
                        self.total, self.total)
        check_pages(dict(table=host(self.table_out), lengths=host(self.lengths_out), copies=host(self.copies), free=host(self.free),
                         left=int(self.left.item()), status=0), want)
        for now, then in zip(self.caches, self.before):
            for source, to, tokens, _ in want["copies"]:
                then[to, :tokens] = then[source, :tokens]
            assert torch.equal(now, then)


def test_captured_steps_replay_on_new_inputs():
    s = Calls()
    s.renew()
    s()
    s.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s()
    for _ in range(4):
        s.renew()
        graph.replay()
        s.check()


def test_marshalled_calls_go_to_the_stream_that_is_current_and_two_searches_do_not_meet():
    a, b = Calls(seed=1), Calls(n=40, beams=7, vocab=777, seed=2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        a.renew(), b.renew()
        torch.cuda.synchronize()
        for _ in range(5):  # the same inputs give the same results again: nothing that is read is written
            for s, stream in zip((a, b), streams):
                with torch.cuda.stream(stream):
                    s.calls[0]()
                    s.calls[1]()
        for s, stream in zip((a, b), streams):
            with torch.cuda.stream(stream):
                s.calls[2]()
        a.check(), b.check()
