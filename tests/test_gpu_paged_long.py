"""Steps over texts of some thousand slots, where attention works in ranges and joins them: in the middle of a workspace of exactly the planned size, captured and
replayed, two graphs with one workspace, two batches on streams of their own, and evictions of as many slots."""
import math

import pytest
import torch

from tests import paged_oracle as oracle

pytestmark = pytest.mark.gpu
HEADS, KV, D, PAGE = 8, 2, 64, 32


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


class Batch:
    def __init__(self, api, lengths, slots, seed, budget):
        g = self.g = torch.Generator().manual_seed(seed)
        n, n_table = len(lengths), -(-slots // PAGE)
        slots = n_table * PAGE
        self.api, self.n, self.slots, self.budget = api, n, slots, budget
        n_pages = n * n_table + 2
        self.table = torch.randperm(n_pages, generator=g)[:n * n_table].view(n, n_table).int()
        k, v = (torch.randn(n_pages, KV, PAGE, D, generator=g).bfloat16() for _ in range(2))
        self.cache = api.Paged(k.cuda(), v.cuda(), self.table.cuda())
        self.lengths, self.after = torch.tensor(lengths, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        self.pos = self.lengths.clone()
        self.weights = torch.rand(n, KV, slots, generator=g).cuda()
        self.positions = torch.stack([torch.arange(slots)] * (n * KV)).view(n, KV, slots).int().cuda()
        self.q, self.o = (torch.zeros(n, HEADS * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.k, self.v = (torch.zeros(n, KV * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.ranges, self.elems = api.tl_k_attention_paged_plan(slots, n, HEADS, KV, D, True, 1 << 30)
        self.evict_elems = n * KV * (2 * max(0, min(budget, slots - budget)) + 1)
        self.ws = torch.full((max(self.elems, self.evict_elems),), math.nan, device="cuda")
        self.inputs()

    def inputs(self):
        for t in (self.q, self.k, self.v):
            t.copy_(torch.randn(*t.shape, generator=self.g))

    def step(self, cut=False):
        api = self.api
        api.tl_k_paged_append(self.cache, self.lengths, self.k, self.v, pos=self.pos, weights=self.weights, positions=self.positions)
        torch.add(self.lengths, 1, out=self.after)
        api.tl_k_attention_paged(self.cache, self.after, self.q, self.o, HEADS, weights_in=self.weights, weights_out=self.weights, workspace=self.ws)
        if cut:
            api.tl_k_paged_evict(self.cache, self.after, self.budget, 100, self.weights, self.positions, self.weights, self.positions, self.lengths, self.ws)
        else:
            self.lengths.copy_(self.after)
        self.pos.add_(1)

    def held(self):
        return (self.cache.k, self.cache.v, self.weights, self.positions, self.lengths, self.pos, self.o)

    def state(self):
        return [t.clone() for t in self.held()]

    def set(self, state):
        for t, x in zip(self.held(), state):
            t.copy_(x)


SHAPES = [([2900, 5, 1411, 0, 3000], 3008, 2000), ([20000], 20032, 9000), ([4100, 37, 35000], 35008, 12000)]


@pytest.mark.parametrize("lengths,slots,budget", SHAPES)
def test_a_workspace_of_exactly_the_planned_size(api, lengths, slots, budget):
    b = Batch(api, lengths, slots, 1, budget)
    assert b.ranges > 1
    for weights in (True, False):
        n, elems = api.tl_k_attention_paged_plan(b.slots, b.n, HEADS, KV, D, weights, 1 << 30)
        assert api.tl_k_attention_paged_plan(b.slots, b.n, HEADS, KV, D, weights, elems) == (n, elems)
        guarded = torch.full((elems + 2048,), -7.25, device="cuda")
        w = torch.full((b.n, KV, b.slots), 5.0, device="cuda") if weights else None
        before = b.lengths.cpu()
        api.tl_k_attention_paged(b.cache, b.lengths, b.q, b.o, HEADS, weights_out=w, workspace=guarded[1024:1024 + elems])
        assert (guarded[:1024] == -7.25).all() and (guarded[1024 + elems:] == -7.25).all()
        assert torch.equal(b.lengths.cpu(), before)
        o, got, tol_o, tol = oracle.attention(b.cache.k.cpu(), b.cache.v.cpu(), b.table, before, b.slots, b.q.cpu(), HEADS)
        # the output's rounding to bf16 (half a step) is of the value with its error
        assert ((b.o.cpu().double() - o).abs() <= tol_o + 2.0 ** -8 * (o.abs() + tol_o)).all()
        if weights:
            for s, m in enumerate(lengths):
                assert (w[s, :, m:] == 5.0).all() and ((w[s, :, :m].cpu().double() - got[s, :, :m]).abs() <= tol[s, :, :m]).all()
    guarded = torch.full((b.evict_elems + 2048,), -7.25, device="cuda")
    api.tl_k_paged_evict(b.cache, b.lengths, budget, 100, b.weights, b.positions, b.weights, b.positions, b.lengths, guarded[1024:1024 + b.evict_elems])
    assert (guarded[:1024] == -7.25).all() and (guarded[1024 + b.evict_elems:] == -7.25).all()
    assert b.lengths.tolist() == [min(n, budget) for n in lengths]


@pytest.mark.parametrize("lengths,slots,budget", SHAPES)
def test_captured(api, lengths, slots, budget):
    """two graphs that use one workspace, replayed in turn with eager steps between them"""
    lengths = [min(n, slots - 40) for n in lengths]
    b = Batch(api, lengths, slots, 2, budget)
    assert b.ranges > 1
    start = b.state()
    b.step(), b.step(True)
    b.set(start)
    graphs, s = [], torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for cut in (False, True):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
            b.step(cut)
        graphs.append(g)
    torch.cuda.current_stream().wait_stream(s)
    b.set(start)
    for i in range(9):
        b.inputs()
        cut, here = i % 3 == 2, b.state()
        b.step(cut)
        want = b.state()
        b.set(here)
        b.ws.fill_(math.nan)
        graphs[cut].replay()
        torch.cuda.synchronize()
        for x, y in zip(b.state(), want):
            assert torch.equal(x, y), i


def test_two_streams(api):
    """two batches with workspaces of their own, at the same time"""
    batches = [Batch(api, [2800, 40, 2000], 3008, 5, 1500), Batch(api, [15000, 14000], 20032, 6, 9000)]
    streams, many, alone = [torch.cuda.Stream() for _ in batches], [], []
    start = [b.state() for b in batches]
    for b in batches:
        rows = []
        for _ in range(8):
            b.inputs()
            rows.append([t.clone() for t in (b.q, b.k, b.v)])
        many.append(rows)

    def run(b, rows):
        for i, row in enumerate(rows):
            for t, x in zip((b.q, b.k, b.v), row):
                t.copy_(x)
            b.step(i % 4 == 3)

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


def test_one_long_text_among_many_short_ones(api):
    """ranges are laid out by the longest: most of them have no key of the others"""
    lengths = [9000] + [1 + 13 * i % 97 for i in range(30)] + [0]
    b = Batch(api, lengths, 9024, 7, 4000)
    assert b.ranges > 1
    w = torch.full((b.n, KV, b.slots), 5.0, device="cuda")
    api.tl_k_attention_paged(b.cache, b.lengths, b.q, b.o, HEADS, weights_out=w, workspace=b.ws)
    o, got, tol_o, tol = oracle.attention(b.cache.k.cpu(), b.cache.v.cpu(), b.table, b.lengths.cpu(), b.slots, b.q.cpu(), HEADS)
    assert ((b.o.cpu().double() - o).abs() <= tol_o + 2.0 ** -8 * (o.abs() + tol_o)).all()
    for s, m in enumerate(lengths):
        assert (w[s, :, m:] == 5.0).all() and ((w[s, :, :m].cpu().double() - got[s, :, :m]).abs() <= tol[s, :, :m]).all()
