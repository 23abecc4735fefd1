"""Which slots an eviction keeps: the order of the header, recent tokens first, among them and among the others larger weights, then lower slots; also where
more tokens are recent than stay, in every form of the kernel that selects."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


def kept_slots(w, p, there, budget, recent):
    """the slots of one head that stay, from lists"""
    newest = max(p)

    def place(j):
        if not there[j]:
            return (0 if j < budget else 3, 0, 0.0, j)
        undefined = w[j] != w[j]
        return (1 if p[j] > newest - recent else 2, undefined, 0.0 if undefined else -w[j], j)
    return set(sorted(range(len(w)), key=place)[:budget])


def run(api, lengths, budget, recent, w, p, table, page, in_place, d=64):
    """checks which token of each head lies in which slot: keys and values say where they come from"""
    n_seqs, kv, width = w.shape
    n_pages = max(int(table.max()) + 1, 1)
    slot = torch.arange(n_pages * page * kv).view(n_pages, kv, page, 1)
    digits = [(slot >> 7 * i & 127).float() for i in range(4)]                 # (whole numbers that bf16 holds)
    k = torch.cat([digits[i % 4] for i in range(d)], dim=3).bfloat16()
    v = (k + 128).bfloat16()
    cache = api.Paged(k.cuda(), v.cuda(), table.cuda())
    gw, gp, L = w.cuda(), p.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    wo, po, Lo = (gw, gp, L) if in_place else (torch.full_like(gw, -9.0), torch.full_like(gp, -9), torch.full_like(L, -9))
    longest = min(width, table.shape[1] * page)
    ws = torch.empty(n_seqs * kv * (2 * max(0, min(budget, longest - budget)) + 1), device="cuda")
    api.tl_k_paged_evict(cache, L, budget, recent, gw, gp, wo, po, Lo, ws)
    assert Lo.tolist() == [min(n, budget) for n in lengths]
    wo, po, k2, v2 = wo.cpu(), po.cpu(), cache.k.cpu(), cache.v.cpu()
    want_k, want_v = k.clone(), v.clone()
    for s, n in enumerate(lengths):
        at = table[s].repeat_interleave(page)[:n]
        there = at >= 0
        off = torch.arange(n) % page
        for h in range(kv):
            stay = torch.zeros(n, dtype=torch.bool)
            stay[list(kept_slots(w[s, h, :n].tolist(), p[s, h, :n].tolist(), there.tolist(), budget, recent) if n > budget else range(n))] = True
            now = torch.arange(min(n, budget))
            hole = ~stay[:budget]
            now[hole] = budget + stay[budget:].nonzero()[:, 0]
            assert torch.equal(po[s, h, :len(now)], p[s, h, now]), (s, h)
            assert torch.equal(wo[s, h, :len(now)].view(torch.int32), w[s, h, now].view(torch.int32)), (s, h)
            to = hole.nonzero()[:, 0]
            fr = now[to]
            assert there[to].all() and there[fr].all()
            for x, y in ((want_k, k), (want_v, v)):
                x[at[to].long(), h, off[to]] = y[at[fr].long(), h, off[fr]]
    assert torch.equal(k2, want_k) and torch.equal(v2, want_v)


def scattered(g, n_seqs, width, page):
    n_table = -(-width // page)
    return torch.randperm(n_seqs * n_table + 2, generator=g)[:n_seqs * n_table].view(n_seqs, n_table).int()


def test_eight_slots(api):
    """positions and weights that rise, 6 recent of which 3 stay: the last three"""
    w, p = torch.arange(8.0)[None, None] + 1, torch.arange(8, dtype=torch.int32)[None, None]
    table = torch.zeros(1, 1, dtype=torch.int32)
    for in_place in (False, True):
        run(api, [8], 3, 6, w, p, table, 16, in_place)
    cache = api.Paged(torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16, device="cuda"), table.cuda())
    wo, po, L = torch.zeros(1, 1, 8, device="cuda"), torch.zeros(1, 1, 8, dtype=torch.int32, device="cuda"), torch.tensor([8], dtype=torch.int32, device="cuda")
    api.tl_k_paged_evict(cache, L, 3, 6, w.cuda(), p.cuda(), wo, po, L, torch.empty(7, device="cuda"))
    assert po[0, 0, :3].tolist() == [5, 6, 7] and wo[0, 0, :3].tolist() == [6.0, 7.0, 8.0]


# widths that each form of the selection takes: 256 threads of 4 slots, 1024 of 4, 8, 16 and 32, and any number read again
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("width", [50, 1024, 1025, 4096, 4099, 8192, 8193, 16384, 16390, 32768, 32769, 40001])
def test_more_recent_than_stay(api, width, in_place):
    """one sequence with more recent tokens than stay beside one with as many, one with fewer, and one that is short"""
    g = torch.Generator().manual_seed(width)
    page, kv = 16, 2
    budget = width // 3
    lengths = [width, budget + 1, width - 1, budget]
    w = torch.rand(4, kv, width, generator=g)
    w[:, 1] = (w[:, 1] * 5).floor()                          # many equals
    p = torch.stack([torch.randperm(width, generator=g) for _ in range(4 * kv)]).view(4, kv, width).int()
    p[2] = torch.arange(width)                               # as they came
    table = scattered(g, 4, width, page)
    for recent in (budget - 1, budget, budget + 1, 2 * budget, 2 ** 31 - 1):
        run(api, lengths, budget, recent, w, p, table, page, in_place)


@pytest.mark.parametrize("width", [300, 4000, 33000])
@pytest.mark.parametrize("recent", [0, 1, 40, 10 ** 9])
def test_equal_positions_and_undefined_weights(api, width, recent):
    """all equally new, or most; undefined, infinite and signed weights among the recent ones; fewer defined ones than stay"""
    g = torch.Generator().manual_seed(width + recent % 1000)
    page, kv, budget = 16, 3, width // 4
    w = torch.randn(4, kv, width, generator=g)
    p = torch.full((4, kv, width), 77, dtype=torch.int32)
    p[1, :, ::3] = 5                                         # a third is older
    p[3] = -2 ** 31                                          # the oldest position there is
    w[1, 0, 1::3] = math.nan                                 # among the recent ones half is undefined
    w[1, 1] = math.nan
    w[1, 2, 1::3], w[1, 2, 2::3] = -math.inf, math.nan
    w[2, 0] = 0.0
    w[2, 0, ::2] = -0.0                                      # (the same value)
    w[2, 1, 7], w[2, 1, width - 1], w[2, 1, 3] = math.inf, math.inf, -math.inf
    w[2, 2] = math.nan
    w[2, 2, width - 20:] = 1e-40                             # a few defined ones, at the end
    run(api, [width] * 4, budget, recent, w, p, scattered(g, 4, width, page), page, False)


@pytest.mark.parametrize("width", [400, 5000, 33000])
def test_more_recent_than_stay_and_pages_that_are_not_there(api, width):
    """slots on no page below the budget stay and take a place each; those behind it are never kept"""
    g = torch.Generator().manual_seed(width)
    page, kv, budget = 16, 2, width // 2
    table = scattered(g, 3, width, page)
    table[0, 2::5] = -1
    table[1, :budget // page - 1] = -1                       # hardly room below the budget
    table[2, budget // page + 1:] = -1                       # few slots on a page behind it
    w = torch.randn(3, kv, width, generator=g)
    w[:, 1, ::4] = math.nan
    p = torch.stack([torch.randperm(width, generator=g) for _ in range(3 * kv)]).view(3, kv, width).int()
    for recent in (budget // 2, budget, width, 2 ** 30):
        run(api, [width] * 3, budget, recent, w, p, table, page, True)
