"""A beam search behind the audio front-end: utterances become log-Mel features (``preba_audio_logmel``), an encoder's states
and their keys and values; a small decoder answers with a beam search over them -- pages, rotation with the cache write,
attention over the cache, attention to the states, selection, block tables of the next beams, copies of their open pages.

    python examples/speech_beam_step.py

The projections are random: the example shows the calls and their buffers, not a model.
"""
from __future__ import annotations

import sys
from pathlib import Path

import numpy as np

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

LAYERS, HEADS_Q, HEADS_KV, DIM, PAGE, VOCAB, STACK, BEGIN, END = 2, 8, 4, 64, 8, 1003, 4, 0, 1
WIDTH = HEADS_Q * DIM


def random(g, *shape):
    """A projection that keeps its input's size."""
    import torch

    return torch.randn(*shape, generator=g, device="cuda").div_(shape[0] ** 0.5).bfloat16()


def encode(utterances, g):
    """States of all utterances, one after the other, and where each one's begin: features of STACK frames, projected."""
    import torch

    from paper_2411_19114_b200 import binding as pb

    packed, table = pb.preba_audio_pack(utterances)
    frames = table["frames"].astype(int)
    mels = torch.empty(len(utterances), pb.AUDIO_MELS, int(frames.max()), dtype=torch.float32, device="cuda")
    pb.preba_audio_logmel(torch.from_numpy(packed).cuda(), torch.from_numpy(table.view(np.uint8)).cuda(), len(utterances),
                          mels.shape[2], mels, table_host=table)
    counts = frames // STACK
    stacked = [mels[i, :, :n * STACK].t().reshape(n, STACK * pb.AUDIO_MELS) for i, n in enumerate(counts)]
    states = torch.cat(stacked).bfloat16() @ random(g, STACK * pb.AUDIO_MELS, WIDTH)
    return states, torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")


class Search:
    """What a server keeps of a batch of searches: tables, lengths, scores, the stack of free pages, the caches, and the layers'
    projections with their keys and values of the states."""

    def __init__(self, states, cu_k, beams: int, longest: int, g):
        import torch

        from paper_2411_19114_b200 import binding as pb

        self.n, self.beams, self.cu_k = cu_k.numel() - 1, beams, cu_k
        rows = self.rows = self.n * beams
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
        width = -(-longest // PAGE) + 1
        self.pages = rows * width + 3
        self.tables = [ints(rows, width).fill_(-1) for _ in range(2)]  # of these beams, and of the next
        self.lengths, self.next_lengths, self.kv_len, self.slots = ints(rows), ints(rows), ints(rows), ints(rows)
        self.fresh, self.cu_q, self.copies = ints(rows).fill_(1), ints(rows + 1), ints(rows, 4)
        self.free, self.free_count, self.free_left = ints(self.pages), ints(1).fill_(self.pages), ints(1)
        self.free.copy_(torch.randperm(self.pages, generator=g, device="cuda"))
        self.status = ints(1)
        # a search begins with one beam; all rows of an utterance see its states
        self.scores = torch.full((self.n, beams), -float("inf"), device="cuda")
        self.scores[:, 0] = 0
        self.next_scores = torch.empty_like(self.scores)
        self.done, self.next_done = (torch.zeros(self.n, beams, dtype=torch.bool, device="cuda") for _ in range(2))
        self.tokens, self.parents = ints(self.n, beams).fill_(BEGIN), ints(self.n, beams)
        self.cu_rows = torch.arange(0, rows + 1, beams, dtype=torch.int32, device="cuda")
        self.embedding = random(g, WIDTH, VOCAB).t().contiguous().mul_(4)
        self.inv_freq = 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64, device="cuda") / (DIM // 2))
        self.qkv = [random(g, WIDTH, (HEADS_Q + 2 * HEADS_KV) * DIM) for _ in range(LAYERS)]
        self.cross_q = [random(g, WIDTH, WIDTH) for _ in range(LAYERS)]
        self.cross_kv = [(states @ random(g, WIDTH, 2 * HEADS_KV * DIM)).view(-1, 2, HEADS_KV, DIM) for _ in range(LAYERS)]
        self.k_caches, self.v_caches = ([torch.zeros(self.pages, PAGE, HEADS_KV, DIM, dtype=torch.bfloat16, device="cuda")
                                         for _ in range(LAYERS)] for _ in range(2))
        bytes_ = lambda size: torch.zeros(size, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.attend_ws = bytes_(pb.preba_pages_attend_query(rows, rows, HEADS_Q, HEADS_KV, DIM))
        self.cross_ws = bytes_(pb.preba_cross_attend_query(self.n, rows, HEADS_Q, HEADS_KV, DIM))
        self.select_ws = bytes_(pb.preba_beam_select_query(self.n, beams, beams, VOCAB, torch.bfloat16))
        self.pages_ws = bytes_(pb.preba_beam_pages_query(self.n, beams, width))

    def step(self):
        """One token for every beam; returns what the step went through, layer by layer, and what it chose."""
        import torch

        from paper_2411_19114_b200 import binding as pb

        table, next_table = self.tables
        trace = dict(tokens=self.tokens.clone(), scores=self.scores.clone(), done=self.done.clone(), layers=[])
        pb.preba_pages_plan(self.lengths, self.fresh, table, self.free, self.free_count, PAGE, self.cu_q, self.kv_len,
                            self.slots, None, self.free_left, pages=self.pages, status=self.status)
        self.free_count.copy_(self.free_left)
        hidden = self.embedding[self.tokens.flatten().long()]
        position = self.lengths[None].expand(3, -1)  # text: the same on all axes
        for layer in range(LAYERS):
            qkv = (hidden @ self.qkv[layer]).view(self.rows, HEADS_Q + 2 * HEADS_KV, DIM)
            q = torch.empty(self.rows, HEADS_Q, DIM, dtype=hidden.dtype, device="cuda")
            own, seen = torch.empty_like(q), torch.empty_like(q)
            pb.preba_rope_append(qkv[:, :HEADS_Q], qkv[:, HEADS_Q:HEADS_Q + HEADS_KV], qkv[:, HEADS_Q + HEADS_KV:], position,
                                 self.inv_freq, (DIM // 2, 0, 0), self.slots, q, self.k_caches[layer], self.v_caches[layer],
                                 status=self.status)
            pb.preba_pages_attend(q, self.k_caches[layer], self.v_caches[layer], table, self.cu_q, self.kv_len, own,
                                  self.attend_ws, max_q=1, scale=DIM ** -0.5, status=self.status)
            asks = (own.flatten(1) @ self.cross_q[layer]).view(self.rows, HEADS_Q, DIM)
            kv = self.cross_kv[layer]
            pb.preba_cross_attend(asks, kv[:, 0], kv[:, 1], self.cu_rows, self.cu_k, seen, self.cross_ws, max_q=self.beams,
                                  scale=DIM ** -0.5, status=self.status)
            trace["layers"].append((qkv, q, own, asks, seen))
            hidden = hidden + own.flatten(1) + seen.flatten(1)
        logits = hidden @ self.embedding.t()
        pb.preba_beam_select(logits, self.scores.flatten(), self.tokens, self.parents, self.next_scores, self.select_ws,
                             end_token=END, done=self.done.flatten(), done_out=self.next_done, status=self.status)
        pb.preba_beam_pages(self.parents, self.kv_len, table, next_table, self.next_lengths, self.copies, self.free,
                            self.free_count, self.free_left, PAGE, self.pages_ws, self.beams, pages=self.pages,
                            status=self.status)
        pb.preba_pages_copy(self.copies, self.k_caches, self.v_caches, status=self.status)
        # the next beams are these now
        self.free_count.copy_(self.free_left)
        self.tables.reverse()
        self.lengths, self.next_lengths = self.next_lengths, self.lengths
        self.scores, self.next_scores = self.next_scores, self.scores
        self.done, self.next_done = self.next_done, self.done
        return dict(trace, logits=logits, chosen=self.tokens.clone(), parents=self.parents.clone(), next_scores=self.scores.clone(),
                    next_done=self.done.clone())


def run(utterances: int = 3, beams: int = 4, steps: int = 20):
    """The search after ``steps`` tokens, and every step's trace."""
    import torch

    from paper_2411_19114_b200 import workloads as wl

    g = torch.Generator(device="cuda").manual_seed(5)
    states, cu_k = encode(wl.utterances(utterances, seed=7, min_s=1.0, max_s=4.0), g)
    search = Search(states, cu_k, beams, steps + 1, g)
    traces = [search.step() for _ in range(steps)]
    torch.cuda.synchronize()
    return search, traces


if __name__ == "__main__":
    searched, done = run()
    print(f"{len(done)} steps of {searched.beams} beams, {searched.cu_k.diff().tolist()} states, scores of the best "
          f"{[round(v, 3) for v in searched.scores[:, 0].tolist()]}, pages left {int(searched.free_count)}, "
          f"status {int(searched.status)}")
