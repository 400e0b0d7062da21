"""What the beam search leaves alone, steps without rows, and the selection's values where nearly all of a row's weight lies far
below its maximum.

Tolerance of the values, counted along the longest way of a term through the sum.  A lane adds 32 elements in four chains (8
additions, the first to zero), joins them (2) and the warp does (5); the product with what the maximum's rounding left is one
more: 15 roundings of 2^-24.  Three exponentials of 2^-22 each (the element's, the left-over's, the segment's) are 12 more.
Their arguments are off by 2^-24 and by 2^-26 (the constant log2 e) of themselves in the element's and by 2 * 2^-24 + 2^-26 in
the segment's; the mean of |x - max| under a softmax is at most its entropy, ln 2^20 < 13.9: 13.9 * 2.25 < 32 more.  59 * 2^-24 <
2^-18, and the value is rounded once.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import beams as ob
from paper_2411_19114_b200 import binding as pb
from test_gpu_beams import DTYPES, check_select, ints, run_select
from test_gpu_cross import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,pad,order", [(64, 8, "nhd"), (8, 8, "hnd"), (80, 48, "nhd"), (128, 64, "hnd")])
def test_copies_leave_what_lies_between_the_heads(d, pad, order, dtype):
    g = torch.Generator(device="cuda").manual_seed(d)
    shape = (9, 16, 3, d + pad) if order == "nhd" else (9, 3, 16, d + pad)
    whole = [torch.randn(shape, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(4)]
    want = [w.clone() for w in whole]
    views = lambda all_: [w[..., :d] if order == "nhd" else w[..., :d].transpose(1, 2) for w in all_]  # noqa: E731
    copies = [[0, 4, 16, 0], [0, 5, 1, 0], [2, 6, 0, 0], [3, 8, 11, 0]]
    for w in views(want):
        for source, to, count, _ in copies:
            w[to, :count] = w[source, :count]
    status, caches = ints([0]), views(whole)
    pb.preba_pages_copy(ints(copies), caches[:2], caches[2:], status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert all(torch.equal(w.view(torch.int16), x.view(torch.int16)) for w, x in zip(whole, want))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("max_q", [1, 300])
@pytest.mark.parametrize("n", [1, 5, 500])
def test_steps_without_rows_write_nothing(n, max_q, d):
    s = Step([4], [50 * n], 4, 2, d, "bf16")
    s.cu_q, s.cu_k = np.full(n + 1, 2), 50 * np.arange(n + 1)
    need = pb.preba_cross_attend_query(n, s.tokens, 4, 2, d)
    s.ws = torch.zeros(need + 64, dtype=torch.uint8, device="cuda")
    s.ws[need:] = 0x5a
    s.need = need
    for _ in range(2):
        s.call(max_q=max_q)
        assert bool((s.out() == 7).all()) and bool((s.lse == 7).all()) and int(s.status.item()) == 0


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("vocab,below", [(1 << 20, 13.75), (200001, 12.25), (32000, 0.0), (1 << 20, 30.0)])
def test_values_where_a_row_is_nearly_flat(vocab, below, dtype):
    x = torch.full((2, vocab), -below, dtype=DTYPES[dtype], device="cuda")
    x[0, vocab // 3], x[1, vocab - 1] = 0, 1.5
    scores = np.array([-0.25, -0.5], dtype=np.float32)
    check_select(run_select(x, scores, 6, 2), ob.select(x.double().cpu().numpy(), scores, 6, 2))
