"""Calls of the serving step that were marshalled once, made again under another stream."""
from __future__ import annotations

import pytest
import torch

from paper_2411_19114_b200 import binding as pb
from test_gpu_tokens import Step, dev

pytestmark = pytest.mark.gpu


def prepared(step, out, stream=None):
    ws = torch.zeros(pb.preba_pages_attend_query(len(step.kv), step.q.shape[0], *step.heads, step.d),
                     dtype=torch.uint8, device="cuda")
    return pb.PreparedPagesAttend(step.q, step.k, step.v, dev(step.table), dev(step.cu), dev(step.kv), out, ws,
                                  max_q=step.max_q, scale=step.scale, stream=stream)


@pytest.mark.parametrize("rows", [1, 30])
def test_a_marshalled_call_goes_to_the_stream_that_is_current(rows):
    step = Step([(300, rows), (77, rows)], 8, 2, 64, 16, seed=9)
    want, _, _ = step.run()
    out = torch.zeros_like(step.q)
    call = prepared(step, out)
    call()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    # captured on a side stream: the call has to be part of the graph
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_a_stream_that_was_named_stays():
    step = Step([(300, 1), (77, 1)], 8, 2, 64, 16, seed=9)
    want, _, _ = step.run()
    out, named, other = torch.zeros_like(step.q), torch.cuda.Stream(), torch.cuda.Stream()
    named.wait_stream(torch.cuda.current_stream())
    call = prepared(step, out, stream=named)
    with torch.cuda.stream(other):
        call()
    named.synchronize()
    assert torch.equal(out, want)
