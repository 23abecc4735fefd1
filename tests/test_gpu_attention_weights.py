"""What a prompt's tokens got of attention, against its definition in 64 bits."""
import math

import pytest
import torch

from tests import paged_oracle as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


def make(seed, T, heads, kv, d):
    g = torch.Generator().manual_seed(seed)
    q, k = torch.randn(T, heads * d, generator=g).bfloat16(), torch.randn(T, kv * d, generator=g).bfloat16()
    lse = torch.empty(heads, T)
    later = torch.ones(T, T, dtype=torch.bool).triu(1)
    for j in range(heads):
        x = q.view(T, heads, d)[:, j].double() @ k.view(T, kv, d)[:, j // (heads // kv)].double().T / math.sqrt(d)
        lse[j] = torch.logsumexp(x.masked_fill(later, -math.inf), dim=1).float()
    return q, k, lse, g


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 130, 500, 777])
@pytest.mark.parametrize("heads,kv,d", [(1, 1, 64), (4, 4, 128), (6, 2, 64), (5, 1, 128)])
def test_column_sums(api, T, heads, kv, d):
    q, k, lse, g = make(T * heads + d, T, heads, kv, d)
    for first in (0, 1, T // 2, T - 1, T, T + 50):
        want, tol = oracle.column_sums(q, k, heads, kv, lse, first)
        out = torch.full((kv, T + 4), 5.0, device="cuda")
        api.tl_k_attention_weights(q.cuda(), k.cuda(), heads, kv, lse.cuda(), None, out, first_row=first)
        assert ((out[:, :T].cpu().double() - want).abs() <= tol).all(), first
        assert (out[:, T:] == 5.0).all()
    w = torch.rand(kv, T, generator=g)
    both = w.cuda()
    api.tl_k_attention_weights(q.cuda(), k.cuda(), heads, kv, lse.cuda(), both, both)
    want, tol = oracle.column_sums(q, k, heads, kv, lse, 0)
    full = w.double() + want
    assert ((both.cpu().double() - full).abs() <= tol + 2.0 ** -24 * full).all()


@pytest.mark.parametrize("T,heads,kv,d", [(2300, 32, 32, 64), (1100, 64, 64, 64), (1500, 64, 64, 128), (3000, 64, 64, 128), (2500, 64, 64, 64), (900, 32, 32, 128),
                                            (2050, 32, 32, 128), (1999, 64, 32, 64), (3001, 64, 32, 128), (4300, 64, 32, 64), (700, 64, 64, 64)])
def test_column_sums_of_many_heads(api, T, heads, kv, d):
    """keys side by side in one, two and four waves, workgroups of four and of eight, blocks alone and in pairs"""
    g = torch.Generator(device="cuda").manual_seed(T)
    q, k = (torch.randn(T, n * d, generator=g, device="cuda").bfloat16() for n in (heads, kv))
    lse = torch.empty(heads, T, device="cuda")
    out = torch.empty(kv, T, device="cuda")
    rows = torch.arange(T, device="cuda")
    want, tol = (torch.zeros(kv, T, dtype=torch.float64, device="cuda") for _ in range(2))
    for j in range(heads):
        h = j // (heads // kv)
        qq, kk = q.view(T, heads, d)[:, j].double(), k.view(T, kv, d)[:, h].double()
        x = (qq @ kk.T / math.sqrt(d)).masked_fill(rows > rows[:, None], -math.inf)
        lse[j] = torch.logsumexp(x, dim=1).float()
        p = torch.exp(x - lse[j].double()[:, None])
        want[h] += p.sum(dim=0)
        size = (qq.abs() @ kk.abs().T / math.sqrt(d)).amax(dim=1, keepdim=True)
        tol[h] += (p * ((d + 3) * 2.0 ** -24 * size + 3 * 2.0 ** -24 * lse[j].double().abs()[:, None] + 2.0 ** -22 + T * 2.0 ** -24)).sum(dim=0)
    api.tl_k_attention_weights(q, k, heads, kv, lse, None, out)
    assert ((out.double() - want).abs() <= tol + heads * 2.0 ** -24 * want).all()


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_rows_anywhere(api, shift):
    T, heads, kv, d = 200, 4, 2, 64
    q, k, lse, _ = make(5, T, heads, kv, d)
    want = torch.empty(kv, T, device="cuda")
    api.tl_k_attention_weights(q.cuda(), k.cuda(), heads, kv, lse.cuda(), None, want)
    for ld in (heads * d + 2 * kv * d, heads * d + 2 * kv * d + 5):
        big = torch.full((T + 1, ld + 8), math.nan, dtype=torch.bfloat16, device="cuda").view(-1)
        rows = big[shift:shift + T * ld].view(T, ld)
        rows[:, :heads * d], rows[:, heads * d:heads * d + kv * d] = q.cuda(), k.cuda()
        out = torch.empty_like(want)
        api.tl_k_attention_weights(rows[:, :heads * d], rows[:, heads * d:heads * d + kv * d], heads, kv, lse.cuda(), None, out)
        assert torch.equal(out, want)


def test_behind_the_prompts_own_attention(api):
    """with the log-sum-exp that it leaves: every row gives away 1 a query head"""
    T, heads, d = 900, 4, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn(T, 3 * heads * d, generator=g, device="cuda").bfloat16()
    q, k, v = (qkv[:, i * heads * d:(i + 1) * heads * d] for i in range(3))
    o, lse, w = torch.empty(T, heads * d, dtype=torch.bfloat16, device="cuda"), torch.empty(heads, T, device="cuda"), torch.empty(heads, T, device="cuda")
    api.tl_k_attention_fwd(q, k, v, heads, d, o, lse)
    api.tl_k_attention_weights(q, k, heads, heads, lse, None, w)
    # T rows, each off by the errors of its scores (below 2^-16) in lse and weights
    assert ((w.double().sum(dim=1) - T).abs() <= T * 2.0 ** -14).all()


def test_an_undefined_row_counts_where_it_is_seen(api):
    T, d = 150, 64
    q, k, lse, _ = make(2, T, 2, 2, d)
    q.view(T, 2, d)[100, 0, 3] = math.nan
    out = torch.empty(2, T, device="cuda")
    api.tl_k_attention_weights(q.cuda(), k.cuda(), 2, 2, lse.cuda(), None, out)
    assert torch.isnan(out[0, :101]).all() and torch.isfinite(out[0, 101:]).all() and torch.isfinite(out[1]).all()
    api.tl_k_attention_weights(q.cuda(), k.cuda(), 2, 2, lse.cuda(), None, out, first_row=101)
    assert torch.isfinite(out).all()
