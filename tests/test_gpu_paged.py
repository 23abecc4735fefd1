"""Append, attention and eviction on a key/value cache on pages, against their definitions in 64 bits."""
import math

import pytest
import torch

from tests import paged_oracle as oracle

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8                       # half a step of bf16, relative


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


def gen(seed):
    return torch.Generator().manual_seed(seed)


def bf16(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).bfloat16()


def pool(g, n_seqs, n_table, kv, page, d, spare=2, k_scale=1.0):
    """pages in a scattered order"""
    n = n_seqs * n_table + spare
    table = torch.randperm(n, generator=g)[:n_seqs * n_table].view(n_seqs, n_table).int()
    return bf16(g, n, kv, page, d, scale=k_scale), bf16(g, n, kv, page, d), table


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def on_gpu(api, k, v, table):
    return api.Paged(k.cuda(), v.cuda(), table.cuda())


# ---------------------------------------------------------------- append
@pytest.mark.parametrize("kv,d,page", [(1, 64, 16), (4, 64, 32), (8, 128, 16), (3, 128, 128), (32, 128, 64)])
def test_append_one_each(api, kv, d, page):
    g = gen(kv * d + page)
    n_seqs, n_table = 6, 3
    k, v, table = pool(g, n_seqs, n_table, kv, page, d)
    table[2, 1], table[3, 0] = -1, k.shape[0]               # no pages
    lengths = ints([0, page - 1, page, 5, n_table * page, -7])
    rk, rv = bf16(g, n_seqs, kv * d), bf16(g, n_seqs, kv * d)
    w, p = torch.randn(n_seqs, kv, n_table * page, generator=g), torch.randint(0, 99, (n_seqs, kv, n_table * page), generator=g).int()
    pos = ints([11, 12, 13, 14, 15, 16])
    cache = on_gpu(api, k, v, table)
    gw, gp = w.cuda(), p.cuda()
    api.tl_k_paged_append(cache, lengths.cuda(), rk.cuda(), rv.cuda(), pos=pos.cuda(), weights=gw, positions=gp)
    oracle.append(k, v, table, lengths, rk, rv, None, pos, w, p)
    for a, b in ((cache.k, k), (cache.v, v), (gw, w), (gp, p)):
        assert torch.equal(a.cpu(), b)


@pytest.mark.parametrize("first_row", [[0, 0, 5, 5, 40, 47], [3, 3, 3, 3, 3, 3], [2, 9, 30, 31, 31, 33], [0, 50, 50, 50, 50, 50]])
def test_append_ragged_strided_and_partly(api, first_row):
    """rows before the first and behind the last sequence are nobody's; weights end inside the table; the table ends inside the rows"""
    g = gen(sum(first_row))
    kv, d, page, n_table, n_rows = 2, 64, 16, 3, 50
    n_seqs = len(first_row) - 1
    k, v, table = pool(g, n_seqs, n_table, kv, page, d)
    table[1, 2] = -5
    lengths = ints([0, 17, 3, 47, 30])
    big = bf16(g, n_rows, 3 * kv * d + 1)
    rk, rv = big[:, 1:1 + kv * d], big[:, 2 * kv * d + 1:]
    w, p = torch.randn(n_seqs, kv, 40, generator=g), torch.zeros(n_seqs, kv, 40, dtype=torch.int32)
    cache = on_gpu(api, k, v, table)
    gb, gw, gp = big.cuda(), w.cuda(), p.cuda()
    api.tl_k_paged_append(cache, lengths.cuda(), gb[:, 1:1 + kv * d], gb[:, 2 * kv * d + 1:], first_row=ints(first_row).cuda(), weights=gw, positions=gp)
    oracle.append(k, v, table, lengths, rk, rv, first_row, None, w, p)
    for a, b in ((cache.k, k), (cache.v, v), (gw, w), (gp, p)):
        assert torch.equal(a.cpu(), b)


# ---------------------------------------------------------------- attention
def check(api, k, v, table, lengths, heads, max_len=None, ws_elems=None, seed=0, q=None, weights=True):
    n_pages, kv, page, d = k.shape
    n_seqs, room = table.shape[0], table.shape[1] * page
    g = gen(seed)
    q = bf16(g, n_seqs, heads * d) if q is None else q
    limit = room if max_len is None else max_len
    o64, got64, tol_o, tol_got = oracle.attention(k, v, table, lengths, limit, q, heads)
    cache = on_gpu(api, k, v, table)
    L = lengths.cuda()
    least = api.tl_k_attention_paged_plan(limit, n_seqs, heads, kv, d, True, 0)[1]
    plans = [None, 1 << 21] if ws_elems is None else [ws_elems]
    outs = []
    for elems in plans:
        ws = None if elems is None else torch.full((max(elems, least),), math.nan, device="cuda")
        o = torch.full((n_seqs, heads * d), 7.0, dtype=torch.bfloat16, device="cuda")
        api.tl_k_attention_paged(cache, L, q.cuda(), o, heads, max_len, workspace=ws)
        outs.append(o.clone())
        if weights and ws is not None:
            w_in = torch.rand(n_seqs, kv, limit + 3, generator=g)
            w_out = torch.full((n_seqs, kv, limit + 3), -3.0, device="cuda")
            o2 = torch.empty_like(o)
            api.tl_k_attention_paged(cache, L, q.cuda(), o2, heads, max_len, w_in.cuda(), w_out, ws)
            assert torch.equal(o2, o)
            same = w_in.cuda()
            api.tl_k_attention_paged(cache, L, q.cuda(), o2, heads, max_len, same, same, ws)
            alone = torch.full_like(w_out, -3.0)
            api.tl_k_attention_paged(cache, L, q.cuda(), o2, heads, max_len, None, alone, ws)
            for s in range(n_seqs):
                n = min(max(int(lengths[s]), 0), limit)
                assert (w_out[s, :, n:] == -3.0).all() and torch.equal(same[s, :, n:].cpu(), w_in[s, :, n:]) and torch.equal(same[s, :, :n], w_out[s, :, :n])
                want, tol = got64[s, :, :n], tol_got[s, :, :n]
                assert ((alone[s, :, :n].cpu().double() - want).abs() <= tol).all(), (s, n)
                full = w_in[s, :, :n].double() + want
                assert ((w_out[s, :, :n].cpu().double() - full).abs() <= tol + 2.0 ** -24 * full.abs()).all(), (s, n)
    for o in outs:
        err = (o.cpu().double() - o64).abs()
        # the output's rounding is of the value with its error
        assert (err <= tol_o + HALF * (o64.abs() + tol_o)).all(), float((err - tol_o - HALF * o64.abs()).max())
    return outs


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (6, 2), (10, 2), (32, 8), (16, 1), (17, 1), (40, 1), (33, 3)])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 32), (128, 64), (64, 256)])
def test_attention(api, heads, kv, d, page):
    g = gen(heads + d + page)
    lengths = ints([0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 250])
    k, v, table = pool(g, len(lengths), -(-256 // page), kv, page, d)
    check(api, k, v, table, lengths, heads, seed=heads)


@pytest.mark.parametrize("lengths", [[1000], [4097], [5000, 3, 2500]])
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 2, 128), (24, 1, 128)])
def test_attention_long(api, lengths, heads, kv, d):
    g = gen(len(lengths) + heads)
    page = 64
    k, v, table = pool(g, len(lengths), -(-max(lengths) // page), kv, page, d, k_scale=2.0)
    check(api, k, v, table, ints(lengths), heads, max_len=max(lengths))
    check(api, k, v, table, ints(lengths), heads, max_len=max(lengths), ws_elems=3 * len(lengths) * heads * (d + 2) + 64, weights=False)


def test_attention_of_large_scores(api):
    """scores up to several hundred: the maximum grows often and far"""
    g = gen(3)
    k, v, table = pool(g, 2, 20, 2, 32, 128, k_scale=30.0)
    k[int(table[0, 9])] *= 4
    check(api, k, v, table, ints([640, 611]), 4)


def test_attention_what_lies_outside_is_not_seen(api):
    """NaN and infinities behind the lengths, on pages that are nobody's, and in place of pages that are not there"""
    g = gen(4)
    kv, d, page, heads = 2, 128, 16, 6
    lengths = ints([5, 40, 100, 64, 0, 96])
    k, v, table = pool(g, 6, 7, kv, page, d)
    table[2, 1], table[2, 5], table[3, :4] = -1, 10 ** 9, -1          # a hole, one more, and no page at all
    table[5, 5] = -2 ** 31
    used = torch.zeros(k.shape[0], page, dtype=torch.bool)
    for s, n in enumerate(lengths.tolist()):
        for j in range(n):
            i = oracle.page_of(table, k.shape[0], s, j, page)
            if i >= 0:
                used[i, j % page] = True
    for x, bad in ((k, math.nan), (v, math.inf)):
        x.masked_fill_(~used[:, None, :, None], bad)
    for o in check(api, k, v, table, lengths, heads):
        assert (o[3] == 0).all() and (o[4] == 0).all()


def test_attention_max_len_cuts(api):
    g = gen(5)
    k, v, table = pool(g, 3, 10, 2, 16, 64)
    for max_len in (1, 16, 37, 160):
        check(api, k, v, table, ints([160, 30, 2 ** 30]), 2, max_len=max_len)


def test_attention_infinite_and_undefined_values(api):
    g = gen(6)
    kv, d, page = 2, 64, 16
    k, v, table = pool(g, 5, 20, kv, page, d)
    lengths = ints([300, 300, 300, 300, 300])
    v[int(table[0, 3]), 1, 2, 7] = math.inf
    v[int(table[1, 18]), 0, 0, 5] = math.nan
    k[int(table[2, 3]), 0, 3] = -math.inf                    # with positive queries: a score of -infinity, a weight of 0
    q = bf16(g, 5, 4 * d).abs()
    k[table[3].long(), 1] = -math.inf                        # nothing but scores of -infinity
    k[int(table[4, 2]), 0, 1] = math.nan
    cache = on_gpu(api, k, v, table)
    for ws in (None, torch.empty(1 << 20, device="cuda")):
        o = torch.empty(5, 4 * d, dtype=torch.bfloat16, device="cuda")
        api.tl_k_attention_paged(cache, lengths.cuda(), q.cuda(), o, 4, workspace=ws)
        o = o.cpu().float().view(5, 2, 2, d)
        assert torch.isinf(o[0, 1, :, 7]).all() and torch.isfinite(o[0, 1, :, :7]).all() and torch.isfinite(o[0, 0]).all()
        assert torch.isnan(o[1, 0, :, 5]).all() and torch.isfinite(o[1, 0, :, 6:]).all()
        assert torch.isfinite(o[2]).all()
        assert torch.isnan(o[3, 1]).all() and torch.isfinite(o[3, 0]).all()
        assert torch.isnan(o[4, 0]).all() and torch.isfinite(o[4, 1]).all()


def test_attention_strided_rows(api):
    g = gen(7)
    kv, d, page, heads, n = 2, 64, 16, 4, 3
    k, v, table = pool(g, n, 4, kv, page, d)
    lengths = ints([64, 20, 33])
    big = bf16(g, n, heads * d + 9)
    cache, gb = on_gpu(api, k, v, table), big.cuda()
    dense, out = torch.empty(n, heads * d, dtype=torch.bfloat16, device="cuda"), torch.full((n, heads * d + 5), 3.0, dtype=torch.bfloat16, device="cuda")
    api.tl_k_attention_paged(cache, lengths.cuda(), gb[:, 3:3 + heads * d].contiguous(), dense, heads)
    api.tl_k_attention_paged(cache, lengths.cuda(), gb[:, 3:3 + heads * d], out[:, 2:2 + heads * d], heads)
    assert torch.equal(out[:, 2:2 + heads * d], dense) and (out[:, :2] == 3).all() and (out[:, 2 + heads * d:] == 3).all()


def test_ranges_reach_what_the_plan_says(api):
    assert api.tl_k_attention_paged_plan(131072, 1, 32, 8, 128, False, 1 << 24)[0] > 16
    assert api.tl_k_attention_paged_plan(200, 1, 4, 4, 64, False, 0) == (1, 0)


def test_pool_beyond_4_gib(api):
    """offsets beyond 2^32 bytes and 2^31 elements"""
    kv, d, page = 8, 128, 64
    n_pages = 36000
    k, v = (torch.zeros(n_pages, kv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 31
    table = torch.tensor([[n_pages - 1, 3, n_pages - 7]], dtype=torch.int32, device="cuda")
    cache = api.Paged(k, v, table)
    g = gen(8)
    rk, rv = bf16(g, 150, kv * d), bf16(g, 150, kv * d)
    api.tl_k_paged_append(cache, ints([0]).cuda(), rk.cuda(), rv.cuda(), first_row=ints([0, 150]).cuda())
    q = bf16(g, 1, 8 * d)
    o = torch.empty(1, 8 * d, dtype=torch.bfloat16, device="cuda")
    api.tl_k_attention_paged(cache, ints([150]).cuda(), q.cuda(), o, 8)
    p = torch.softmax(torch.einsum("hd,jhd->hj", q.view(8, d).double(), rk.view(150, 8, d).double()) / math.sqrt(d), dim=1)
    want = torch.einsum("hj,jhd->hd", p, rv.view(150, 8, d).double()).view(1, -1)
    size = torch.einsum("hj,jhd->hd", p, rv.view(150, 8, d).double().abs()).view(1, -1)
    assert ((o.cpu().double() - want).abs() <= HALF * want.abs() + 2.0 ** -12 * size).all()
    w, pos = torch.rand(1, kv, 150, generator=g).cuda(), torch.arange(150, dtype=torch.int32).expand(1, kv, 150).contiguous().cuda()
    small_k, small_v = (x[table[0].long()].cpu() for x in (k, v))
    after, w64, p64 = oracle.evict(small_k, small_v, ints([[0, 1, 2]]), ints([150]), 70, 20, w.cpu(), pos.cpu())
    L = ints([150]).cuda()
    api.tl_k_paged_evict(cache, L, 70, 20, w, pos, w, pos, L, torch.empty(kv * 141, device="cuda"))
    assert L.tolist() == [70] and torch.equal(k[table[0].long()].cpu(), small_k) and torch.equal(v[table[0].long()].cpu(), small_v)
    assert torch.equal(pos.cpu(), p64) and int((k[10:n_pages - 8] != 0).sum()) == 0


# ---------------------------------------------------------------- eviction
def evict_case(g, lengths, kv, page, d, room=None):
    n_seqs = len(lengths)
    n_table = -(-max(max(lengths), 1, room or 1) // page)
    k, v, table = pool(g, n_seqs, n_table, kv, page, d)
    width = n_table * page
    w = torch.exp(2 * torch.randn(n_seqs, kv, width, generator=g))
    p = torch.stack([torch.randperm(width, generator=g) for _ in range(n_seqs * kv)]).view(n_seqs, kv, width).int()
    return k, v, table, w, p


def check_evict(api, k, v, table, lengths, budget, recent, w, p, in_place):
    cache = on_gpu(api, k, v, table)
    n_seqs, kv = table.shape[0], k.shape[1]
    width = min(w.shape[2], table.shape[1] * k.shape[2])
    ws = torch.empty(n_seqs * kv * (2 * max(0, min(budget, width - budget)) + 1), device="cuda")
    L, gw, gp = lengths.cuda(), w.cuda(), p.cuda()
    wo, po = (gw, gp) if in_place else (torch.full_like(gw, -9.0), torch.full_like(gp, -9))
    Lo = L if in_place else torch.full_like(L, -9)
    api.tl_k_paged_evict(cache, L, budget, recent, gw, gp, wo, po, Lo, ws)
    after, w2, p2 = oracle.evict(k, v, table, lengths, budget, recent, w, p)
    assert torch.equal(Lo.cpu(), after)
    assert torch.equal(cache.k.cpu().view(torch.int16), k.view(torch.int16)) and torch.equal(cache.v.cpu().view(torch.int16), v.view(torch.int16))
    for s, n in enumerate(after.tolist()):
        assert torch.equal(po[s, :, :n].cpu(), p2[s, :, :n]) and torch.equal(wo[s, :, :n].cpu().view(torch.int32), w2[s, :, :n].view(torch.int32)), s
        if not in_place:
            assert (wo[s, :, n:] == -9).all() and (po[s, :, n:] == -9).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lengths,budget,recent", [([1], 1, 0), ([2, 1, 0], 1, 1), ([33, 17, 16], 16, 5), ([300, 120, 0, 299, 65], 100, 30), ([300, 120], 100, 100), ([300], 100, 500),
                                                   ([300], 299, 10), ([300], 300, 10), ([300, 4], 500, 0), ([1025, 2050], 1024, 7), ([3000], 50, 0), ([5000], 4000, 1999)])
def test_evict(api, lengths, budget, recent, in_place):
    g = gen(sum(lengths) + budget)
    k, v, table, w, p = evict_case(g, lengths, 3, 16, 64)
    check_evict(api, k, v, table, ints(lengths), budget, recent, w, p, in_place)


@pytest.mark.parametrize("kv,page,d", [(1, 64, 128), (8, 32, 128), (5, 128, 64)])
def test_evict_layouts(api, kv, page, d):
    g = gen(kv)
    k, v, table, w, p = evict_case(g, [700, 333, 512], kv, page, d)
    check_evict(api, k, v, table, ints([700, 333, 512]), 256, 64, w, p, True)


def test_evict_equal_undefined_and_signed_weights(api):
    g = gen(9)
    k, v, table, w, p = evict_case(g, [400] * 6, 2, 16, 64)
    w[0] = 0.0                                                # all equal: the lowest slots stay
    w[0, 1, ::2] = -0.0                                       # (the same value)
    w[1] = math.nan
    w[1, 0, 300:310] = 1.0
    w[2] = torch.randint(0, 3, (2, 400), generator=g).float()[:, :w.shape[2]]
    w[3] = -w[3]
    w[4, 0, 17], w[4, 0, 399], w[4, 1, 5] = math.inf, math.inf, -math.inf
    p[5] = 77                                                 # all of them the newest
    for recent in (0, 1, 40):
        check_evict(api, k.clone(), v.clone(), table, ints([400] * 6), 120, recent, w, p, False)


def test_evict_pages_that_are_not_there_and_short_rows(api):
    g = gen(10)
    k, v, table, w, p = evict_case(g, [400, 390, 250], 2, 16, 64)
    table[0, 3], table[0, 20], table[1, 5:20], table[2, 10] = -1, 10 ** 6, -1, -1
    check_evict(api, k.clone(), v.clone(), table, ints([400, 390, 250]), 200, 50, w, p, False)
    # hardly more slots on pages than stay, and fewer
    table[0, 1:14] = -1
    check_evict(api, k.clone(), v.clone(), table, ints([400, 390, 250]), 200, 50, w, p, False)
    table[0, 14:20] = -1
    check_evict(api, k.clone(), v.clone(), table, ints([400, 390, 250]), 200, 50, w, p, True)
    # weights for fewer slots than the table has room for: lengths count as that
    check_evict(api, k, v, table, ints([400, 390, 250]), 200, 50, w[:, :, :300].contiguous(), p[:, :, :300].contiguous(), True)


@pytest.mark.parametrize("n,budget", [(8191, 3000), (8192, 100), (8193, 5000), (8195, 8194), (20001, 4096), (32768, 4096), (32769, 9000), (40003, 39000)])
def test_evict_of_many_slots(api, n, budget):
    """slots held by 256 and by 1024 threads, and read again; with many equal weights"""
    g = gen(n)
    kv, page, d = 2, 64, 64
    n_table = -(-n // page)
    k, v = (bf16(g, n_table, kv, page, d) for _ in range(2))
    table = torch.randperm(n_table, generator=g)[None].int()
    w = torch.rand(1, kv, n, generator=g)
    w[0, 1] = (w[0, 1] * 4).floor()
    p = torch.randperm(n, generator=g)[None, None].expand(1, kv, n).int().contiguous()
    cache = on_gpu(api, k, v, table)
    for recent in (0, budget // 3):
        key = torch.where(p > p.max() - recent, math.inf, w)
        order = torch.sort(key, dim=2, descending=True, stable=True).indices[0, :, :budget]
        wo, po = torch.zeros(1, kv, n, device="cuda"), torch.zeros(1, kv, n, dtype=torch.int32, device="cuda")
        c = on_gpu(api, k, v, table)
        L = torch.zeros(1, dtype=torch.int32, device="cuda")
        most = max(0, min(budget, min(n, n_table * page) - budget))
        api.tl_k_paged_evict(c, ints([n]).cuda(), budget, recent, w.cuda(), p.cuda(), wo, po, L, torch.empty(kv * (2 * most + 1), device="cuda"))
        assert L.tolist() == [budget]
        for h in range(kv):
            kept = torch.zeros(n, dtype=torch.bool)
            kept[order[h]] = True
            now = torch.arange(budget)
            now[~kept[:budget]] = budget + kept[budget:].nonzero()[:, 0]
            assert torch.equal(wo[0, h, :budget].cpu(), w[0, h, now]) and torch.equal(po[0, h, :budget].cpu(), p[0, h, now])
            slots = torch.arange(n)
            slots[:budget] = now
            for x, y in ((c.k, k), (c.v, v)):
                at = table[0].long()
                got = x.cpu()[at, h].reshape(-1, d)[:n]
                assert torch.equal(got, y[at, h].reshape(-1, d)[slots])


def test_evict_of_many_slots_with_pages_that_are_not_there(api):
    g = gen(12)
    kv, page, d, n, budget = 1, 16, 64, 33000, 20000
    n_table = -(-n // page)
    k, v = (bf16(g, n_table, kv, page, d) for _ in range(2))
    table = torch.randperm(n_table, generator=g)[None].int()
    table[0, torch.randperm(n_table, generator=g)[:300]] = -1
    w, p = torch.rand(1, kv, n, generator=g), torch.randperm(n, generator=g)[None, None].int()
    for m in (n, 30000):                                     # read again, and held in registers
        check_evict(api, k.clone(), v.clone(), table, ints([m]), budget, 500, w[:, :, :m].contiguous(), p[:, :, :m].contiguous(), False)
