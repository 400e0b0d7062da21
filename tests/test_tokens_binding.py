"""What the binding of the serving step takes and refuses, with host tensors that say they are on a GPU:
nothing is launched."""
from __future__ import annotations

import pytest
import torch

from paper_2411_19114_b200 import binding as pb
from test_tokens_boundary import built_library  # noqa: F401


class OnGpu(torch.Tensor):
    """A host tensor that says it is on a GPU."""

    @property
    def is_cuda(self):
        return True


def gpu(t):
    return t.as_subclass(OnGpu)


def ints(*shape):
    return gpu(torch.zeros(shape, dtype=torch.int32))


def halves(*shape):
    return gpu(torch.zeros(shape, dtype=torch.float16))


def plan(**other):
    return pb.PreparedPagesPlan(**{**dict(
        cached=ints(2), fresh=ints(2), block_table=ints(2, 4), free_pages=ints(8), free_count=ints(1), page_size=16,
        cu_q=ints(3), kv_len=ints(2), slots=ints(5), positions=ints(5), free_left=ints(1), pages=64, status=ints(1),
        stream=0), **other})


def positions(**other):
    return pb.PreparedRopePositions(**{**dict(
        spans=ints(3, 4), span_begin=ints(3), cached=ints(2), cu_q=ints(3), positions=ints(3, 5), status=ints(1),
        stream=0), **other})


def append(**other):
    return pb.PreparedRopeAppend(**{**dict(
        q=halves(5, 4, 64), k=halves(5, 2, 64), v=halves(5, 2, 64), positions=ints(3, 5),
        inv_freq=gpu(torch.zeros(32, dtype=torch.float64)), sections=(16, 8, 8), slots=ints(5), q_out=halves(5, 4, 64),
        k_cache=halves(4, 16, 2, 64), v_cache=halves(4, 16, 2, 64), status=ints(1), stream=0), **other})


def attend(**other):
    return pb.PreparedPagesAttend(**{**dict(
        q=halves(5, 4, 64), k_cache=halves(4, 16, 2, 64), v_cache=halves(4, 16, 2, 64), block_table=ints(2, 4),
        cu_q=ints(3), kv_len=ints(2), out=halves(5, 4, 64), workspace=gpu(torch.zeros(4096, dtype=torch.uint8)),
        max_q=4, scale=0.125, lse=gpu(torch.zeros(5, 4)), status=ints(1), stream=0), **other})


def test_good_operands_are_taken():
    for call in (plan, positions, append, attend):
        call()
        call(status=None)
    plan(positions=None)
    attend(lse=None)


@pytest.mark.parametrize("call", [plan, positions, append, attend])
def test_a_status_that_the_kernels_cannot_write_is_refused(call):
    for wrong in (torch.zeros(1, dtype=torch.int32), ints(2), ints(0), gpu(torch.zeros(1, dtype=torch.int64)),
                  gpu(torch.zeros(1))):
        with pytest.raises(ValueError, match="status"):
            call(status=wrong)


def test_a_workspace_or_lse_on_the_host_is_refused():
    for wrong in (torch.zeros(4096, dtype=torch.uint8), gpu(torch.zeros(4096, 2, dtype=torch.uint8))[:, 0]):
        with pytest.raises(ValueError, match="workspace"):
            attend(workspace=wrong)
    for wrong in (torch.zeros(5, 4), gpu(torch.zeros(4, 5)).t(), gpu(torch.zeros(5, 4, dtype=torch.float64))):
        with pytest.raises(ValueError, match="lse"):
            attend(lse=wrong)


def test_operands_on_different_devices_are_refused():
    for call in (plan, positions, append, attend):
        with pytest.raises(ValueError, match="devices"):
            call(status=gpu(torch.zeros(1, dtype=torch.int32, device="meta")))


def test_the_stream_is_the_one_that_is_current_at_the_call(monkeypatch):
    current, used = [11], []
    monkeypatch.setattr(pb, "_current_stream", lambda: lambda device: current[0])
    for make in (plan, positions, append, attend):
        for stream, want in ((None, [11, 12]), (77, [77, 77])):
            call, current[0] = make(stream=stream), 11
            call._call = lambda struct, at: used.append(getattr(at, "value", at)) or pb.OK
            call()
            current[0] = 12
            call()
            assert used[-2:] == want
