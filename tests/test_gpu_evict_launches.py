"""Evictions of as many sequences and slots as one launch has to take: what moves needs a workgroup for each 32 pairs, and a launch has fewer than 2^32 threads."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


@pytest.mark.parametrize("n_seqs,kv,budget,width", [(8192, 8, 8192, 16384), (16384, 16, 2048, 4096), (8191, 8, 8192, 16384)])
def test_many_sequences_with_room_for_many_pairs(api, n_seqs, kv, budget, width):
    """rows * ceil(budget / 32) = 2^24 workgroups and about as many; few sequences are longer than the budget, on pages of their own"""
    g = torch.Generator().manual_seed(n_seqs)
    page, d = width // 4, 64
    long_ones = {0: budget + 1, 77: width, n_seqs - 1: budget + 40}
    table = torch.full((n_seqs, 4), -1, dtype=torch.int32)
    for i, s in enumerate(long_ones):
        table[s] = torch.arange(4 * i, 4 * i + 4)
    k, v = (torch.randn(12, kv, page, d, generator=g).bfloat16() for _ in range(2))
    w, p = torch.zeros(n_seqs, kv, width, device="cuda"), torch.zeros(n_seqs, kv, width, dtype=torch.int32, device="cuda")
    for s in long_ones:
        w[s] = torch.rand(kv, width, generator=g).cuda()
        p[s] = torch.stack([torch.randperm(width, generator=g) for _ in range(kv)]).int().cuda()
    before_w, before_p = ({s: t[s].cpu() for s in long_ones} for t in (w, p))
    lengths = torch.arange(n_seqs, dtype=torch.int32) % 7
    for s, n in long_ones.items():
        lengths[s] = n
    cache, L = api.Paged(k.cuda(), v.cuda(), table.cuda()), lengths.cuda()
    recent = budget // 2
    api.tl_k_paged_evict(cache, L, budget, recent, w, p, w, p, L, torch.empty(n_seqs * kv * (2 * min(budget, width - budget) + 1), device="cuda"))
    assert torch.equal(L.cpu(), lengths.clamp(max=budget))
    after = [x.cpu() for x in (cache.k, cache.v)]
    for i, (s, n) in enumerate(long_ones.items()):
        for h in range(kv):
            bw, bp = before_w[s][h, :n], before_p[s][h, :n]
            key = torch.where(bp > int(bp.max()) - recent, 2.0 + bw.double(), bw.double())       # (weights lie below 1)
            order = torch.sort(key, descending=True, stable=True).indices[:budget]
            stay = torch.zeros(n, dtype=torch.bool)
            stay[order] = True
            now = torch.arange(budget)
            now[~stay[:budget]] = budget + stay[budget:].nonzero()[:, 0]
            assert torch.equal(w[s, h, :budget].cpu(), bw[now]) and torch.equal(p[s, h, :budget].cpu(), bp[now])
            for x, y in zip(after, (k, v)):
                was, got = (t[4 * i:4 * i + 4, h].reshape(-1, d) for t in (y, x))
                assert torch.equal(got[:budget], was[now]) and torch.equal(got[budget:], was[budget:])
    others = torch.ones(n_seqs, dtype=torch.bool, device="cuda")
    others[list(long_ones)] = False
    assert not w[others].any() and not p[others].any()
