"""A serving step behind the preprocessing front-end: images that arrive with prompts are resized,
cropped and normalised (``preba_preprocess``), cut into patches and projected to tokens, and one
attention layer over a paged cache takes the whole prompts first and single tokens after that --
pages, positions, rotation with the cache write, attention.

    python examples/image_prompt_step.py

The projections are random: the example shows the calls and their buffers, not a model.
"""
from __future__ import annotations

import sys
from pathlib import Path

import numpy as np

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

PATCH, PAGE, HEADS_Q, HEADS_KV, DIM = 14, 16, 8, 2, 64
WIDTH = HEADS_Q * DIM


class Layer:
    """One attention layer's projections and its part of the paged cache."""

    def __init__(self, pages: int, seed: int = 0):
        import torch

        g = torch.Generator(device="cuda").manual_seed(seed)
        self.qkv = torch.randn(WIDTH, (HEADS_Q + 2 * HEADS_KV) * DIM, generator=g, device="cuda").div_(WIDTH ** 0.5)
        self.qkv = self.qkv.bfloat16()
        self.k_cache, self.v_cache = (
            torch.zeros(pages, PAGE, HEADS_KV, DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))


class Server:
    """What a server keeps between steps: the stack of free pages, the block table, the lengths."""

    def __init__(self, requests: int, pages: int, width: int):
        import torch

        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
        self.n = requests
        self.table = ints(requests, width).fill_(-1)
        self.free = torch.randperm(pages, device="cuda").to(torch.int32)
        self.free_count, self.free_left = ints(1).fill_(pages), ints(1)
        self.cached = ints(requests)
        self.cu_q, self.kv_len, self.status = ints(requests + 1), ints(requests), ints(1)
        self.layer = Layer(pages)
        self.inv_freq = 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64, device="cuda") / (DIM // 2))
        self.sections = (DIM // 2 - 2 * (DIM // 8), DIM // 8, DIM // 8)

    def step(self, hidden, fresh, spans, span_begin):
        """One layer over the step's rows: hidden [tokens, WIDTH] of ``fresh`` rows per request."""
        import torch

        from paper_2411_19114_b200 import binding as pb

        tokens, max_q = hidden.shape[0], int(max(fresh))
        rows = torch.tensor(fresh, dtype=torch.int32, device="cuda")
        slots = torch.empty(tokens, dtype=torch.int32, device="cuda")
        positions = torch.empty(3, tokens, dtype=torch.int32, device="cuda")
        pb.preba_pages_plan(self.cached, rows, self.table, self.free, self.free_count, PAGE, self.cu_q,
                            self.kv_len, slots, None, self.free_left,
                            pages=self.layer.k_cache.shape[0], status=self.status)
        pb.preba_rope_positions(spans, span_begin, self.cached, self.cu_q, positions, status=self.status)
        qkv = (hidden @ self.layer.qkv).view(tokens, HEADS_Q + 2 * HEADS_KV, DIM)
        q = torch.empty(tokens, HEADS_Q, DIM, dtype=hidden.dtype, device="cuda")
        pb.preba_rope_append(qkv[:, :HEADS_Q], qkv[:, HEADS_Q:HEADS_Q + HEADS_KV], qkv[:, HEADS_Q + HEADS_KV:],
                             positions, self.inv_freq, self.sections, slots, q, self.layer.k_cache,
                             self.layer.v_cache, status=self.status)
        out = torch.empty_like(q)
        workspace = torch.zeros(pb.preba_pages_attend_query(self.n, tokens, HEADS_Q, HEADS_KV, DIM),
                                dtype=torch.uint8, device="cuda")
        pb.preba_pages_attend(q, self.layer.k_cache, self.layer.v_cache, self.table, self.cu_q, self.kv_len,
                              out, workspace, max_q=max_q, scale=DIM ** -0.5, status=self.status)
        # the step is over: what was fresh is cached, what was taken from the stack is gone.  A request
        # that was refused (status; its kv_len is 0) keeps its tokens and pages and can be tried again
        self.cached.copy_(torch.where(self.kv_len > 0, self.kv_len, self.cached))
        self.free_count.copy_(self.free_left)
        return q, out, positions, slots


def run(requests: int = 3, new_tokens: int = 4):
    """The prompts of ``requests`` requests with an image each, then ``new_tokens`` single tokens;
    returns the server and every step's (hidden, q, out, positions, slots)."""
    import torch

    from paper_2411_19114_b200 import binding as pb
    from paper_2411_19114_b200 import workloads as wl

    images = wl.mixed_smooth(requests, seed=11)
    packed, table = pb.preba_pack(images)
    pixels = torch.empty(requests, 3, wl.OUT_SIZE, wl.OUT_SIZE, dtype=torch.bfloat16, device="cuda")
    pb.preba_preprocess(torch.from_numpy(packed).cuda(), torch.from_numpy(table.view(np.uint8)).cuda(), requests,
                        pixels, wl.OUT_SIZE, wl.RESIZE_SHORT, wl.MEAN, wl.STD, pb.BF16, table_host=table)
    side = wl.OUT_SIZE // PATCH
    patches = torch.nn.functional.unfold(pixels.float(), PATCH, stride=PATCH).transpose(1, 2)  # [n, side^2, 3*14*14]
    g = torch.Generator(device="cuda").manual_seed(1)
    project = torch.randn(patches.shape[2], WIDTH, generator=g, device="cuda").div_(patches.shape[2] ** 0.5)
    # every prompt: some text, the image, some more text
    text = [(5 + 7 * r, 3 + r) for r in range(requests)]
    spans, prompts = [], []
    for r, (before, after) in enumerate(text):
        spans += [(before, 0, 0, 1), (1, side, side, 1), (after, 0, 0, 1)]
        words = torch.randn(before + after, WIDTH, generator=g, device="cuda")
        prompts.append(torch.cat([words[:before], patches[r] @ project, words[before:]]))
    spans = torch.tensor(spans, dtype=torch.int32, device="cuda")
    span_begin = torch.arange(0, 3 * requests + 1, 3, dtype=torch.int32, device="cuda")
    longest = max(p.shape[0] for p in prompts) + new_tokens
    server = Server(requests, pages=requests * (longest // PAGE + 2), width=longest // PAGE + 1)

    steps = []
    fresh = [p.shape[0] for p in prompts]
    hidden = torch.cat(prompts).bfloat16()
    for _ in range(1 + new_tokens):
        q, out, positions, slots = server.step(hidden, fresh, spans, span_begin)
        steps.append((hidden, q, out, positions, slots))
        # the last row of each request stands in for the next token's embedding
        last = server.cu_q[1:].long() - 1
        hidden, fresh = out.flatten(1)[last].contiguous(), [1] * requests
    torch.cuda.synchronize()
    return server, steps


if __name__ == "__main__":
    served, done = run()
    print(f"{len(done)} steps, {[s[0].shape[0] for s in done]} rows, keys per request "
          f"{served.kv_len.tolist()}, pages left {int(served.free_left)}, status {int(served.status)}")
