"""One request, one token, one head or one page, in tensors whose axis of that one entry has an odd
stride: nothing steps along it, so it is no reason to refuse the call."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2411_19114_b200 import binding as pb
from test_gpu_tokens import Step, dev, new_status

pytestmark = pytest.mark.gpu


def odd(t, axis):
    """The same entries, with a stride of 1 on an axis that has one."""
    assert t.shape[axis] == 1
    strides = list(t.stride())
    strides[axis] = 1
    return t.as_strided(t.shape, strides)


@pytest.mark.parametrize("rows", [1, 30])
def test_attention(rows):
    step = Step([(14, rows)] if rows == 1 else [(64, rows)], 4, 1, 64, 64, seed=rows)
    page = int(step.table[0, 0])
    step.k, step.v = step.k[page:page + 1].clone(), step.v[page:page + 1].clone()
    step.table = np.zeros((1, 5), dtype=np.int64)
    want, want_lse, status = step.run()
    assert status == 0
    k, v = odd(odd(step.k, 0), 2), odd(odd(step.v, 0), 2)
    q = odd(step.q, 0) if rows == 1 else step.q
    out, lse, status = torch.zeros_like(want), torch.zeros(rows, 4, device="cuda"), new_status()
    ws = torch.zeros(pb.preba_pages_attend_query(1, rows, 4, 1, 64), dtype=torch.uint8, device="cuda")
    pb.preba_pages_attend(q, k, v, odd(dev(step.table), 0), dev(step.cu), dev(step.kv), out, ws, max_q=rows,
                          scale=step.scale, lse=lse, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and torch.equal(out, want) and np.array_equal(lse.cpu().numpy(), want_lse)


def test_plan_and_rotation():
    table, ints = dev(np.full((1, 5), -1)), lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    slots, cu, kv, left, status = ints(1), ints(2), ints(1), ints(1), new_status()
    pb.preba_pages_plan(dev([0]), dev([1]), odd(table, 0), dev([0]), dev([1]), 16, cu, kv, slots, None, left, pages=1,
                        status=status)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(1, 1, 64, generator=g, device="cuda").half()
    caches = [torch.zeros(1, 16, 1, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
    out, pos = torch.zeros_like(x), dev(np.zeros((3, 1)))
    inv = torch.ones(32, dtype=torch.float64, device="cuda")
    pb.preba_rope_append(odd(x, 0), odd(x, 1), x, pos, inv, (16, 8, 8), slots, odd(out, 1), odd(caches[0], 0),
                         odd(caches[1], 2), status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and table.tolist() == [[0, -1, -1, -1, -1]] and kv.tolist() == [1]
    assert torch.equal(out, x) and all(torch.equal(c[0, 0], x[0]) and float(c[0, 1:].abs().sum()) == 0 for c in caches)
