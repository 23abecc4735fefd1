"""Counts of tokens, and penalties, bias and mask on logits with the greedy choice, against their definitions in 64 bits."""
import math

import pytest
import torch

from tests import cache8_oracle as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


def gen(seed):
    return torch.Generator().manual_seed(seed)


@pytest.mark.parametrize("rows,n,vocab", [(1, 0, 5), (1, 1, 1), (1, 5000, 32000), (3, 77, 8192), (5, 300, 8193), (2, 1000, 50001), (130, 65, 100),
                                          (64, 4500, 33000), (300, 70, 500), (1, 30000, 9000)])
def test_counts(api, rows, n, vocab):
    tok = torch.randint(-3, vocab + 3, (rows, n), generator=gen(n + vocab), dtype=torch.int32)
    if n > 4:
        tok[0, :3] = torch.tensor([2 ** 31 - 1, -2 ** 31, vocab], dtype=torch.int32)
    want = torch.zeros(rows, vocab, dtype=torch.int32)
    for r in range(rows):
        t = tok[r][(tok[r] >= 0) & (tok[r] < vocab)].long()
        want[r] = torch.bincount(t, minlength=vocab).int()
    buf = torch.full((rows, vocab + 3), -7, dtype=torch.int32, device="cuda")
    counts = buf[:, :vocab]
    api.tl_k_token_counts(tok.cuda(), counts)
    assert torch.equal(counts.cpu(), want)
    api.tl_k_token_counts(tok.cuda(), counts, add=1)
    assert torch.equal(counts.cpu(), 2 * want)
    api.tl_k_token_counts(tok.cuda(), counts, add=-1)
    assert torch.equal(counts.cpu(), want) and (buf[:, vocab:] == -7).all()


def test_counts_of_one_id(api):
    tok = torch.full((2, 20000), 6, dtype=torch.int32, device="cuda")
    c = torch.empty(2, 9, dtype=torch.int32, device="cuda")
    for add, n in ((0, 20000), (1, 40000)):
        api.tl_k_token_counts(tok, c, add=add)
        assert c[:, 6].tolist() == [n, n] and int(c.sum()) == 2 * n


def inputs(rows, vocab, seed, shared):
    g = gen(seed)
    one = 1 if shared else rows
    logits = torch.randn(rows, vocab, generator=g) * 5
    counts = (torch.randint(0, 6, (one, vocab), generator=g) - 3).clamp(min=0).int()
    bias = torch.randn(one, vocab, generator=g) * (torch.rand(one, vocab, generator=g) < 0.3)
    allowed = torch.randint(-2 ** 31, 2 ** 31, (one, (vocab + 31) // 32), generator=g).int()
    return logits, counts, bias, allowed


def dev(t):
    if t is None:
        return None
    return t[0].cuda() if t.shape[0] == 1 else t.cuda()


def check(api, logits, counts, bias, allowed, rep, pres, freq, workspace):
    R, V = logits.shape
    out = torch.full((R, V), 9.0, device="cuda")
    choice = torch.full((R,), -9, dtype=torch.int32, device="cuda")
    api.tl_k_choose(logits.cuda(), dev(counts), out, choice, rep, pres, freq, dev(bias), dev(allowed), workspace)
    f = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    want, may = oracle.choose(logits, counts, f(rep), f(pres), f(freq), bias, allowed)
    got = out.cpu().double()
    # at most four roundings of values no larger than |x| rep + |penalty| + |bias|
    size = logits.double().abs() * max(f(rep), 1 / f(rep)) + abs(f(pres))
    if counts is not None:
        size = size + abs(f(freq)) * counts.double()
    if bias is not None:
        size = size + bias.double().abs()
    assert torch.equal(got == -math.inf, want == -math.inf)
    fin = torch.isfinite(want)
    assert ((got - want).abs()[fin] <= 5 * 2.0 ** -24 * size.expand(R, V)[fin]).all()
    # of the kernel's own values: the largest allowed, the lowest index
    for r in range(R):
        c = int(choice[r])
        ok = may[r] & ~torch.isnan(got[r])
        if not ok.any():
            assert c == -1
        else:
            top = got[r][ok].max()
            assert c == int((ok & (got[r] == top)).nonzero()[0]), r


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 31), (1, 33), (1, 1000), (1, 32000), (3, 2048), (3, 2049), (40, 5003), (200, 776), (20, 32000), (17, 40001)])
@pytest.mark.parametrize("shared", [False, True])
def test_choose(api, rows, vocab, shared):
    logits, counts, bias, allowed = inputs(rows, vocab, rows * vocab, shared)
    ws = torch.full((1 << 18,), math.nan, device="cuda")
    for w in (None, ws):
        check(api, logits, counts, bias, allowed, 1.3, 0.4, 0.07, w)
    check(api, logits, None, bias, allowed, 1.3, 0.4, 0.07, ws)
    check(api, logits, counts, None, allowed, 0.8, -0.2, 0.0, ws)
    check(api, logits, counts, bias, None, 1.0, 0.0, 1.5, ws)
    check(api, logits, None, None, None, 1.0, 0.0, 0.0, ws)


@pytest.mark.parametrize("vocab", [100, 40000])
@pytest.mark.parametrize("with_workspace", [False, True])
def test_equal_nan_infinite_and_no_values(api, vocab, with_workspace):
    ws = torch.full((1 << 16,), math.nan, device="cuda") if with_workspace else None
    x = torch.zeros(7, vocab)
    x[0, [vocab // 2, vocab - 1]] = 3.0                      # two equal: the lower index
    x[1] = math.nan                                          # nothing but NaN
    x[2] = math.nan
    x[2, vocab - 2] = -5.0                                   # one number among NaN
    x[3] = -math.inf                                         # all -infinity: the first allowed
    x[4, 70] = math.inf
    x[5, 99] = 100.0                                         # not allowed
    allowed = torch.full((7, (vocab + 31) // 32), -1, dtype=torch.int32)
    allowed[3, 0] = ~0b111
    allowed[5, 3] = ~(1 << 3)
    allowed[6] = 0                                           # nothing allowed
    out = torch.empty(7, vocab, device="cuda")
    choice = torch.empty(7, dtype=torch.int32, device="cuda")
    api.tl_k_choose(x.cuda(), None, out, choice, allowed=allowed.cuda(), workspace=ws)
    assert choice.tolist() == [vocab // 2, -1, vocab - 2, 3, 70, 0, -1]
    assert (out[6] == -math.inf).all() and torch.isnan(out[1]).all()


def test_bits_behind_the_vocabulary_are_not_read_as_tokens(api):
    x = torch.arange(40.0).view(1, 40).cuda()
    allowed = torch.tensor([[0, -1]], dtype=torch.int32, device="cuda")     # tokens 32 .. 39, and bits that stand for none
    choice = torch.empty(1, dtype=torch.int32, device="cuda")
    api.tl_k_choose(x, None, None, choice, allowed=allowed)
    assert int(choice) == 39


def test_in_place_strided_and_parts(api):
    rows, vocab = 5, 3001
    logits, counts, bias, allowed = inputs(rows, vocab, 3, False)
    ws = torch.empty(1 << 16, device="cuda")
    out = torch.empty(rows, vocab, device="cuda")
    choice = torch.empty(rows, dtype=torch.int32, device="cuda")
    args = dict(repetition=1.1, presence=0.2, frequency=0.3, bias=bias.cuda(), allowed=allowed.cuda())
    api.tl_k_choose(logits.cuda(), counts.cuda(), out, choice, workspace=ws, **args)
    for w in (None, ws):
        buf = torch.full((rows, vocab + 9), 4.0, device="cuda")
        x = buf[:, 3:3 + vocab]
        x.copy_(logits)
        again = torch.empty_like(choice)
        api.tl_k_choose(x, counts.cuda(), x, again, workspace=w, **args)
        assert torch.equal(x, out) and torch.equal(again, choice)
        assert (buf[:, :3] == 4.0).all() and (buf[:, 3 + vocab:] == 4.0).all()
        again.fill_(-5)
        api.tl_k_choose(logits.cuda(), counts.cuda(), None, again, workspace=w, **args)
        assert torch.equal(again, choice)
        other = torch.zeros_like(out)
        api.tl_k_choose(logits.cuda(), counts.cuda(), other, None, workspace=w, **args)
        assert torch.equal(other, out)


def test_plain_choice_is_the_argmax(api):
    x = torch.randn(1, 32000, generator=gen(1)).cuda()
    a, b = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    api.tl_k_argmax(x, a)
    api.tl_k_choose(x, None, None, b, workspace=torch.empty(1 << 12, device="cuda"))
    assert int(a) == int(b)


def test_captured_choice(api):
    rows, vocab = 3, 32000
    logits, counts, bias, allowed = (t.cuda() for t in inputs(rows, vocab, 5, False))
    tok = torch.randint(0, vocab, (rows, 50), generator=gen(6), dtype=torch.int32).cuda()
    ws, out = torch.empty(1 << 16, device="cuda"), torch.empty(rows, vocab, device="cuda")
    choice = torch.empty(rows, dtype=torch.int32, device="cuda")

    def step():
        api.tl_k_token_counts(tok, counts)
        api.tl_k_choose(logits, counts, out, choice, 1.2, 0.1, 0.2, bias, allowed, ws)

    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    for i in range(3):
        logits.copy_(torch.randn(rows, vocab, generator=gen(20 + i)))
        step()
        want = out.clone(), choice.clone(), counts.clone()
        out.zero_(), choice.zero_(), counts.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(choice, want[1]) and torch.equal(counts, want[2])
