"""Calls over lists that overlap on the GPU, each with a scratch of its own: graphs replayed on streams of their own beside eager calls
on a third one; and calls of every kind one behind the other on one stream without a synchronisation, each reading what the
one before wrote.  Every result is that of the call alone, bit for bit."""
import math
import random

import pytest
import torch

from paper_2609_37001_b200 import binding as B
from test_attn_lists import SCALE, pack, random_lists, tensors
from test_select_blocks import blocks_of_tokens

pytestmark = pytest.mark.gpu


def test_graphs_and_an_eager_call_at_once():
    grid, tile, heads = (6, 32, 48), (1, 16, 16), 30
    nb = blocks_of_tokens(grid, tile)[1]
    q, k, v = tensors(heads, math.prod(grid), 13)
    jobs = []
    for seed in (1, 2, 3):
        lists = pack(random_lists(heads, nb, seed, "ragged"))
        want = B.psa_attn_fwd_lists(q, k, v, *lists, grid, tile, SCALE)
        assert B.psa_last_attn_launch()[:2] == (heads * nb, "ticket")   # planned: items and a ticket in the scratch
        got = [torch.empty_like(x) for x in want]
        scratch = torch.empty(B.psa_attn_fwd_lists_scratch_bytes(heads, grid, tile), dtype=torch.uint8, device="cuda")
        jobs.append((torch.cuda.Stream(), lists, want, got, scratch))

    def call(job):
        _, lists, _, (out, lse), scratch = job
        B.psa_attn_fwd_lists(q, k, v, *lists, grid, tile, SCALE, out=out, lse=lse, scratch=scratch)

    graphs = []
    for job in jobs[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(job)
    runs = [g.replay for g in graphs] + [lambda: call(jobs[2])]
    for n in range(6):
        for job in jobs:
            for x in job[3]:
                x.zero_()
        for job in jobs:
            job[0].wait_stream(torch.cuda.current_stream())
        for i in range(3):
            for _ in range(2):   # (the second one of a stream behind its first, beside the others)
                with torch.cuda.stream(jobs[(i + n) % 3][0]):
                    runs[(i + n) % 3]()
        torch.cuda.synchronize()
        assert B.psa_last_device_status() == (0, 0)
        for job in jobs:
            assert all(torch.equal(a, b) for a, b in zip(job[3], job[2]))


KINDS = {   # mode: grid, tile, heads, kind of lists, text tokens
    "shared_direct": ((8, 16, 16), (2, 8, 16), 2, "all", 0),
    "direct": ((4, 16, 16), (1, 16, 16), 30, "one", 0),
    "ticket": ((3, 16, 48), (1, 16, 16), 40, "ragged", 0),
    "ticket_short": ((4, 32, 48), (1, 8, 16), 20, "ragged", 0),
    "ticket padded": ((3, 15, 45), (1, 16, 16), 40, "ragged", 9),
    "ticket_short padded": ((4, 31, 47), (1, 8, 16), 20, "ragged", 0),
}


class Layer:
    """Norm and rotation in place, choice of blocks, attention over the chosen ones, then over other lists, the stripes' launch in between."""

    def __init__(self, kind):
        self.grid, self.tile, self.heads, lists, self.text = KINDS[kind]
        self.n = math.prod(self.grid)
        self.q, self.k, self.v = tensors(self.heads, self.n + self.text, 17)
        self.nb = blocks_of_tokens(self.grid, self.tile)[1]
        self.lists = pack(random_lists(self.heads, self.nb, 18, lists))
        self.params = [((2, 0, 0, 3, 0, 0), (1, 0, 0, 1, 0, 0), (1, 1, 0, 2, 0, 0))[h % 3] for h in range(self.heads)]
        self.keep = (self.nb + 2) // 3
        self.state = [torch.empty_like(x) for x in (self.q, self.k)]
        self.chosen = (torch.empty(self.heads * self.nb + 1, dtype=torch.int32, device="cuda"),
                       torch.empty(self.heads * self.nb * self.keep, dtype=torch.int32, device="cuda"))
        self.scratch = torch.empty(B.psa_attn_fwd_lists_scratch_bytes(self.heads, self.grid, self.tile, self.text), dtype=torch.uint8, device="cuda")
        self.select_scratch = torch.empty(B.psa_select_scratch_bytes(self.heads, self.grid, self.tile), dtype=torch.uint8, device="cuda")
        self.out = [[torch.empty_like(self.q), torch.empty(self.q.shape[:2], device="cuda")] for _ in range(3)]

    def steps(self):
        q, k = self.state
        video = [x[:, :self.n] for x in self.state]
        how = dict(n_text=self.text, scratch=self.scratch)
        return [
            lambda: [a.copy_(b) for a, b in zip(self.state, (self.q, self.k))],
            lambda: B.psa_qk_norm_rope(q, k, self.grid, n_text=self.text, out=(q, k)),
            lambda: B.psa_select_blocks(*video, self.grid, self.tile, self.keep, out=self.chosen, scratch=self.select_scratch),
            lambda: B.psa_attn_fwd_lists(q, k, self.v, *self.chosen, self.grid, self.tile, SCALE, out=self.out[0][0], lse=self.out[0][1], **how),
            lambda: B.psa_attn_fwd_lists(q, k, self.v, *self.lists, self.grid, self.tile, SCALE, out=self.out[1][0], lse=self.out[1][1], **how),
            lambda: B.psa_attn_fwd_joint(q, k, self.v, self.params, self.grid, self.tile, SCALE, self.text, out=self.out[2][0], lse=self.out[2][1]),
            lambda: B.psa_qk_norm_rope(self.out[0][0], None, self.grid, n_text=self.text, norm="token", out=(q, None)),
            lambda: [x.fill_(-3) for x in (k, *self.chosen)],
        ]

    def results(self):
        return [x.clone() for x in (self.state[0], *self.out[0], *self.out[1], *self.out[2])]


def test_in_a_row():
    layers, want = [Layer(kind) for kind in KINDS], []
    for layer, kind in zip(layers, KINDS):
        for i, step in enumerate(layer.steps()):
            step()
            if i == 4:
                assert B.psa_last_attn_launch()[1] == kind.split()[0]
            torch.cuda.synchronize()
        want.append(layer.results())
    rng = random.Random(1)
    for _ in range(8):
        for layer in layers:
            for x in (x for pair in layer.out for x in pair):
                x.fill_(9)
        torch.cuda.synchronize()
        # every layer's steps in their order, those of the layers among one another
        left = {i: layer.steps() for i, layer in enumerate(layers)}
        while left:
            i = rng.choice(sorted(left))
            for _ in range(rng.randint(1, 4)):
                if left[i]:
                    left[i].pop(0)()
            if not left[i]:
                del left[i]
        torch.cuda.synchronize()
        assert B.psa_last_device_status() == (0, 0)
        for layer, expected in zip(layers, want):
            assert all(torch.equal(a, b) for a, b in zip(layer.results(), expected))
