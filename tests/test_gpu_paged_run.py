"""The calls on a cache on pages as one generation makes them, eagerly and captured: a batch of prompts, steps that append, attend, keep what each token got,
cut back, and draw."""
import math

import pytest
import torch

from tests import paged_oracle as oracle

pytestmark = pytest.mark.gpu
HEADS, KV, D, PAGE, TABLE, V = 8, 2, 64, 16, 6, 300


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


class Batch:
    """buffers of one batch, whose tensors a captured graph goes on using"""

    def __init__(self, api, n, seed):
        g = self.g = torch.Generator().manual_seed(seed)
        new = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
        self.api, self.n = api, n
        n_pages = n * TABLE + 1
        table = torch.randperm(n_pages, generator=g)[:n * TABLE].view(n, TABLE).int().cuda()
        self.cache = api.Paged(new(n_pages, KV, PAGE, D, dtype=torch.bfloat16), new(n_pages, KV, PAGE, D, dtype=torch.bfloat16), table)
        self.before, self.after = new(n, dtype=torch.int32), new(n, dtype=torch.int32)
        self.pos = new(n, dtype=torch.int32)
        self.weights, self.positions = new(n, KV, TABLE * PAGE), new(n, KV, TABLE * PAGE, dtype=torch.int32)
        self.q, self.o = new(n, HEADS * D, dtype=torch.bfloat16), new(n, HEADS * D, dtype=torch.bfloat16)
        self.k, self.v = new(n, KV * D, dtype=torch.bfloat16), new(n, KV * D, dtype=torch.bfloat16)
        self.head = (torch.randn(HEADS * D, V, generator=g) * 0.3).cuda()
        self.logits, self.u, self.choice = new(n, V), new(n), new(n, dtype=torch.int32)
        self.params = torch.tensor([0.9, 40, 0.95, 0.01], device="cuda")
        elems = max(api.tl_k_attention_paged_plan(TABLE * PAGE, n, HEADS, KV, D, True, 0)[1], n * KV * (2 * 40 + 1))
        self.ws = torch.full((elems + 20000,), math.nan, device="cuda")

    def inputs(self):
        for t in (self.q, self.k, self.v):
            t.copy_(torch.randn(*t.shape, generator=self.g))
        self.u.copy_(torch.rand(self.n, generator=self.g))

    def prompts(self, lengths):
        api, first = self.api, [0]
        for n in lengths:
            first.append(first[-1] + n)
        q, k, v = ((torch.randn(first[-1], w, generator=self.g)).bfloat16().cuda() for w in (HEADS * D, KV * D, KV * D))
        pos = torch.cat([torch.arange(n) for n in lengths]).int().cuda()
        api.tl_k_paged_append(self.cache, self.before, k, v, torch.tensor(first, dtype=torch.int32, device="cuda"), pos, self.weights, self.positions)
        for s, n in enumerate(lengths):
            a, b = first[s], first[s + 1]
            lse, o = torch.empty(HEADS, n, device="cuda"), torch.empty(n, HEADS * D, dtype=torch.bfloat16, device="cuda")
            kk, vv = (x[a:b].view(n, KV, 1, D).expand(n, KV, HEADS // KV, D).reshape(n, HEADS * D) for x in (k, v))
            qkv = torch.cat([q[a:b], kk, vv], dim=1)
            parts = [qkv[:, i * HEADS * D:(i + 1) * HEADS * D] for i in range(3)]
            api.tl_k_attention_fwd(*parts, HEADS, D, o, lse)
            api.tl_k_attention_weights(q[a:b], k[a:b], HEADS, KV, lse, self.weights[s], self.weights[s])
        self.before.copy_(torch.tensor(lengths, dtype=torch.int32))
        self.pos.copy_(self.before)

    def step(self, cut):
        api = self.api
        api.tl_k_paged_append(self.cache, self.before, self.k, self.v, pos=self.pos, weights=self.weights, positions=self.positions)
        torch.add(self.before, 1, out=self.after)
        api.tl_k_attention_paged(self.cache, self.after, self.q, self.o, HEADS, weights_in=self.weights, weights_out=self.weights, workspace=self.ws)
        if cut:
            api.tl_k_paged_evict(self.cache, self.after, 40, 10, self.weights, self.positions, self.weights, self.positions, self.before, self.ws)
        else:
            self.before.copy_(self.after)
        self.pos.add_(1)
        torch.mm(self.o.float(), self.head, out=self.logits)
        api.tl_k_sample(self.logits, self.params, self.u, self.choice)

    def state(self):
        return [t.clone() for t in (self.cache.k, self.cache.v, self.weights, self.positions, self.before, self.pos, self.o, self.logits, self.choice)]

    def set(self, state):
        for t, x in zip((self.cache.k, self.cache.v, self.weights, self.positions, self.before, self.pos, self.o, self.logits, self.choice), state):
            t.copy_(x)


def test_a_generation_by_its_definitions(api):
    b = Batch(api, 3, 1)
    b.prompts([30, 1, 57])
    for i in range(25):
        b.inputs()
        c = b.cache
        k, v, table, before, w, p = (t.cpu() for t in (c.k, c.v, c.table, b.before, b.weights, b.positions))
        cut = i % 6 == 5
        b.step(cut)
        oracle.append(k, v, table, before, b.k.cpu(), b.v.cpu(), None, b.pos.cpu() - 1, w, p)
        o, got, tol_o, tol = oracle.attention(k, v, table, before + 1, TABLE * PAGE, b.q.cpu(), HEADS)
        assert ((b.o.cpu().double() - o).abs() <= tol_o + 2.0 ** -8 * (o.abs() + tol_o)).all(), i
        full = w.double() + got
        if cut:
            # (by the weights that the step gave, which the next comparison holds to their definition: eviction goes by exact comparisons)
            seen = torch.where(torch.arange(TABLE * PAGE) < (before + 1)[:, None, None], full, w.double())
            after, w2, p2 = oracle.evict(k, v, table, before + 1, 40, 10, seen, p)
            assert torch.equal(b.before.cpu(), after)
            full = w2.double()
            tol = tol.amax(dim=2, keepdim=True).expand_as(tol)
            p = p2
        for s in range(3):
            n = int(b.before[s])
            assert torch.equal(b.positions[s, :, :n].cpu(), p[s, :, :n]), (i, s)
            assert ((b.weights[s, :, :n].cpu().double() - full[s, :, :n]).abs() <= tol[s, :, :n] + 2.0 ** -24 * full[s, :, :n].abs()).all(), (i, s)
        for a, x in ((c.k, k), (c.v, v)):
            assert torch.equal(a.cpu(), x), i
        assert b.choice.tolist() == oracle.sample(b.logits.cpu(), b.params.cpu().expand(3, 4), b.u.cpu())[0]


def test_captured_steps(api):
    b = Batch(api, 4, 2)
    b.prompts([12, 50, 3, 33])
    b.inputs()
    b.step(False)
    graphs, s = [], torch.cuda.Stream()
    start = b.state()
    s.wait_stream(torch.cuda.current_stream())
    for cut in (False, True):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
            b.step(cut)
        graphs.append(g)
    torch.cuda.current_stream().wait_stream(s)
    b.set(start)
    for i in range(12):
        b.inputs()
        here = b.state()
        b.step(i % 4 == 3)                                     # eagerly
        want = b.state()
        b.set(here)
        graphs[i % 4 == 3].replay()
        torch.cuda.synchronize()
        for x, y in zip(b.state(), want):
            assert torch.equal(x, y), i


def test_two_streams(api):
    """two batches with workspaces of their own, at the same time"""
    batches = [Batch(api, 5, 3), Batch(api, 5, 4)]
    streams = [torch.cuda.Stream() for _ in batches]
    for b in batches:
        b.prompts([20, 60, 1, 33, 48])
    many = []
    for b in batches:
        rows = []
        for _ in range(10):
            b.inputs()
            rows.append([t.clone() for t in (b.q, b.k, b.v, b.u)])
        many.append(rows)
    start = [b.state() for b in batches]

    def run(b, rows):
        for i, row in enumerate(rows):
            for t, x in zip((b.q, b.k, b.v, b.u), row):
                t.copy_(x)
            b.step(i % 5 == 4)

    alone = []
    for b, rows in zip(batches, many):
        run(b, rows)
        alone.append(b.state())
    for b, x in zip(batches, start):
        b.set(x)
    torch.cuda.synchronize()
    for s, b, rows in zip(streams, batches, many):
        with torch.cuda.stream(s):
            run(b, rows)
    torch.cuda.synchronize()
    for b, want in zip(batches, alone):
        for x, y in zip(b.state(), want):
            assert torch.equal(x, y)
