"""The 8-bit key/value cache and attention over it against their definitions in 64 bits."""
import math

import pytest
import torch

from tests import cache8_oracle as oracle

pytestmark = pytest.mark.gpu
HI_LO = 2.0 ** -16        # a probability as two bf16 parts: what is left of the second, half a step of 2^-8 of at most 2^-8
BF16 = 2.0 ** -8


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


def draw(seed, n, heads, d, big=4.0):
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(n, heads, d, generator=g)
    k[..., ::16] *= big
    return k.view(n, heads * d).bfloat16(), torch.randn(n, heads * d, generator=g).bfloat16()


def fill(api, k, v, heads, capacity=None, pieces=None):
    """a cache of these rows, everything else in it NaN or codes of 127"""
    n, d = k.shape[0], k.shape[1] // heads
    c = api.Cache8.empty(heads, d, capacity or n)
    for name, t in c.tensors.items():
        t.fill_(127 if t.dtype == torch.int8 else math.nan)
    at = 0
    for m in pieces or [n]:
        api.tl_k_cache8_append(c, at, k[at:at + m].cuda(), v[at:at + m].cuda())
        at += m
    assert at == n
    return c


def read(api, c, n_cached, first, n):
    w = c.n_kv_heads * c.d_head
    out = [torch.full((n, w), math.nan, device="cuda") for _ in range(2)]
    api.tl_k_cache8_read(c, n_cached, first, *out)
    return [x.cpu() for x in out]


def same(a, b):
    return torch.equal(a.view(torch.int32), b.view(torch.int32))


@pytest.mark.parametrize("heads,d", [(1, 64), (3, 128), (4, 64), (2, 128)])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 128, 200, 577])
def test_append_and_read_are_exact(api, n, heads, d):
    k, v = draw(n * 7 + heads, n, heads, d)
    c = fill(api, k, v, heads, capacity=n + 5)
    for x, got in zip((k, v), read(api, c, n, 0, n)):
        assert same(got.view(n, heads, d), oracle.held(x, heads)[0])
    full = n // 64
    for x, name in ((k, "k"), (v, "v")):
        _, codes, scales = oracle.held(x, heads)
        assert same(c.tensors[name + "_scale"][:full].cpu(), scales)
        t = c.tensors[name][:full].cpu().float()
        t = t.permute(0, 3, 1, 2, 4).reshape(full * 64, heads, d) if name == "k" else t.permute(0, 3, 1, 2).reshape(full * 64, heads, d)
        assert torch.equal(t, codes)


@pytest.mark.parametrize("pieces", [[1] * 131, [63, 1, 64, 3], [10, 100, 21], [64, 67], [65, 66], [131]])
def test_cache_does_not_depend_on_the_calls(api, pieces):
    heads, d, n = 2, 64, 131
    k, v = draw(3, n, heads, d)
    whole = fill(api, k, v, heads)
    parts = fill(api, k, v, heads, pieces=pieces)
    for a, b in zip(read(api, whole, n, 0, n), read(api, parts, n, 0, n)):
        assert same(a, b)
    for name in ("k", "v"):
        assert torch.equal(whole.tensors[name][:2], parts.tensors[name][:2])


def test_read_of_a_range(api):
    heads, d, n = 2, 128, 300
    k, v = draw(4, n, heads, d)
    c = fill(api, k, v, heads, capacity=320)
    everything = read(api, c, n, 0, n)
    for first, m in ((0, 1), (63, 2), (64, 64), (100, 190), (255, 45), (256, 44), (299, 1), (300, 0)):
        for a, b in zip(everything, read(api, c, n, first, m)):
            assert same(a[first:first + m], b)


def test_codes_at_the_borders_of_two(api):
    """quotients that are exact ties, or next to one; the smallest and largest magnitudes; zeros"""
    d, rows = 64, []
    for top in (127.0, 1.0, 254.0, 96.0, 2.0 ** -90, 2.0 ** -99, 2.0 ** 100, 3.3e38, 2.0 ** -110, 1e-40, 0.0):
        s = max(top, 2.0 ** -100) / 127
        # half-way points, rounded to bf16, and their neighbours
        base = ((torch.arange(64)[:, None] * 2 - 127 + torch.arange(d)[None] % 3 * 0.5) * s).bfloat16()
        bits = (base.view(torch.int16).int() + torch.arange(d)[None] % 5 - 2).to(torch.int16)
        t = torch.nan_to_num(bits.view(torch.bfloat16).float(), nan=0.0).clamp(-top, top).bfloat16()     # (below zero's bits are NaN's)
        t[0, 0] = top
        rows.append(t)
    x = torch.cat(rows)
    assert torch.isfinite(x).all()
    c = fill(api, x, x.flip(1).contiguous(), 1)
    got = read(api, c, len(x), 0, len(x))
    assert same(got[0].view(-1, 1, d), oracle.held(x, 1)[0])
    assert same(got[1].view(-1, 1, d), oracle.held(x.flip(1).contiguous(), 1)[0])


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_block_with_a_value_that_is_not_finite(api, bad):
    heads, d, n = 2, 64, 200
    k, v = draw(5, n, heads, d)
    k[70, 3] = bad             # block 1, head 0
    v[130, d + 5] = bad        # block 2, head 1
    v[195, 7] = bad            # tail, head 0
    c = fill(api, k, v, heads)
    for x, got in zip((k, v), read(api, c, n, 0, n)):
        want = oracle.held(x, heads)[0].view(n, -1)
        assert torch.equal(torch.isnan(want), torch.isnan(got))
        assert torch.equal(torch.nan_to_num(want, 0.0), torch.nan_to_num(got, 0.0))


def test_append_of_strided_and_misaligned_rows(api):
    heads, d, n = 3, 64, 150
    k, v = draw(6, n, heads, d)
    want = read(api, fill(api, k, v, heads), n, 0, n)
    buf = torch.full((n * 700 + 8,), math.nan, dtype=torch.bfloat16, device="cuda")
    for off in (0, 1, 2, 3):
        both = buf[off:off + n * 700].view(n, 700)
        kk, vv = both[:, 5:5 + heads * d], both[:, 301:301 + heads * d]
        kk.copy_(k), vv.copy_(v)
        c = api.Cache8.empty(heads, d, n)
        api.tl_k_cache8_append(c, 0, kk[:77], vv[:77])
        api.tl_k_cache8_append(c, 77, kk[77:], vv[77:])
        for a, b in zip(want, read(api, c, n, 0, n)):
            assert same(a, b)


# ---------------------------------------------------------------- attention
def attend(api, c, n, q, heads, workspace=None):
    o = torch.full_like(q, math.nan).cuda()
    api.tl_k_attention_cache8(c, n, q.cuda(), o, heads, workspace)
    return o.cpu()


def check(api, c, n, k, v, q, heads, kv, workspace=None, p_rounding=None):
    d = c.d_head
    if p_rounding is None:
        name = api.tl_k_attention_cache8_plan(n, q.shape[0], heads, kv, d, 0 if workspace is None else workspace.numel())[0]
        p_rounding = HI_LO if name.startswith("columns") else BF16
    got = attend(api, c, n, q, heads, workspace).double().view(q.shape[0], heads, d)
    want, size, reach = oracle.attention(q, oracle.held(k[:n], kv)[0], oracle.held(v[:n], kv)[0], heads)
    far = (got - want).abs() - oracle.attention_bound(want, size, reach, d, n, p_rounding)
    assert torch.isfinite(got).all() and far.max() <= 0, (far.max(), n, q.shape)


def queries(seed, rows, width):
    return torch.randn(rows, width, generator=torch.Generator().manual_seed(seed)).bfloat16()


@pytest.mark.parametrize("heads,kv,d", [(1, 1, 64), (4, 4, 128), (6, 2, 64), (8, 1, 128), (20, 1, 64)])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 128, 130, 257, 512, 700, 705, 1500, 3333])
def test_one_row(api, n, heads, kv, d):
    k, v = draw(n + heads, n, kv, d)
    c = fill(api, k, v, kv, capacity=n + 70)
    q = queries(n, 1, heads * d)
    for ws in (None, torch.full((1 << 18,), math.nan, device="cuda")):
        check(api, c, n, k, v, q, heads, kv, ws)


@pytest.mark.parametrize("heads,kv,d", [(2, 2, 64), (4, 1, 128), (3, 3, 128)])
@pytest.mark.parametrize("rows,n", [(2, 2), (3, 64), (5, 66), (16, 80), (17, 300), (33, 33), (64, 128), (65, 200), (100, 129), (200, 200)])
def test_rows(api, rows, n, heads, kv, d):
    k, v = draw(n + rows, n, kv, d)
    c = fill(api, k, v, kv, capacity=n + 1)
    q = queries(n, rows, heads * d)
    for ws in (None, torch.full((1 << 18,), math.nan, device="cuda")):
        check(api, c, n, k, v, q, heads, kv, ws)


@pytest.mark.parametrize("heads,kv,d,rows,n", [
    (1, 1, 64, 300, 301), (1, 1, 128, 256, 512), (2, 2, 128, 257, 400), (6, 2, 64, 90, 700), (8, 1, 128, 33, 500), (8, 1, 64, 130, 131),
    (1, 1, 128, 700, 700), (16, 16, 64, 140, 300), (16, 16, 128, 257, 321), (16, 16, 64, 300, 300), (3, 1, 64, 11, 4000), (5, 1, 128, 13, 2500), (2, 2, 64, 40, 63), (4, 4, 128, 100, 2063)])
def test_many_columns(api, heads, kv, d, rows, n):
    k, v = draw(n + rows, n, kv, d)
    c = fill(api, k, v, kv, capacity=n + 1)
    q = queries(n, rows, heads * d)
    for ws in (None, torch.full((1 << 20,), math.nan, device="cuda")):
        check(api, c, n, k, v, q, heads, kv, ws)


# keys, rows, heads, key heads, d; the last two are more workgroups than run at once
WIDE = [(600, 520, 64, 64, 64), (1000, 600, 32, 32, 64), (600, 520, 64, 64, 128), (1300, 260, 32, 32, 128), (450, 390, 250, 250, 128), (600, 550, 160, 160, 64)]


@pytest.mark.parametrize("n,rows,heads,kv,d", WIDE)
@pytest.mark.parametrize("elems", [0, 1 << 22])
def test_many_columns_of_many_heads(api, n, rows, heads, kv, d, elems):
    k, v = draw(n + rows, n, kv, d)
    c = fill(api, k, v, kv, capacity=n + 1)
    q = queries(n, rows, heads * d)
    got = attend(api, c, n, q, heads, torch.full((elems,), math.nan, device="cuda") if elems else None).double().view(rows, heads, d).cuda()
    kh, vh = (oracle.held(x, kv)[0].double().cuda().transpose(0, 1) for x in (k, v))
    later = torch.arange(n, device="cuda")[None] > torch.arange(rows, device="cuda")[:, None] + n - rows
    for h in range(heads):
        qh = q.view(rows, heads, d)[:, h].double().cuda()
        p = torch.softmax((qh @ kh[h].T / math.sqrt(d)).masked_fill(later, -math.inf), 1)
        want, size = p @ vh[h], p @ vh[h].abs()
        reach = (qh.abs() @ kh[h].abs().T).amax(1, keepdim=True) / math.sqrt(d)
        far = (got[:, h] - want).abs() - oracle.attention_bound(want, size, reach, d, n, BF16)
        assert far.max() <= 0, (h, far.max())


def test_every_kernel_is_reached(api):
    """by the sizes above, with and without ranges"""
    sizes = [(66, 5, 2, 2, 64), (257, 1, 4, 4, 128), (200, 65, 2, 2, 64), (4000, 11, 3, 1, 64), (2063, 100, 4, 4, 128), WIDE[0], WIDE[1]]
    seen = {api.tl_k_attention_cache8_plan(*s, elems)[0] for s in sizes for elems in (0, 1 << 20, 1 << 22)}
    assert seen == {"columns8", "columns16", "rows128", "rows256"}


def test_ranges_with_nothing_to_see(api):
    """more ranges than the first rows reach: their part of the join is empty"""
    heads, d, n, rows = 1, 64, 2000, 1000
    k, v = draw(8, n, heads, d)
    c = fill(api, k, v, heads)
    q = queries(1, rows, heads * d)
    ws = torch.full((1 << 22,), math.nan, device="cuda")
    check(api, c, n, k, v, q, heads, heads, ws)


def test_many_ranges_and_a_small_workspace(api):
    heads, kv, d, n = 4, 2, 64, 5000
    k, v = draw(9, n, kv, d)
    c = fill(api, k, v, kv)
    q = queries(2, 1, heads * d)
    per = heads * (d + 2)
    counts = set()
    for elems in (1, per, 2 * per - 1, 2 * per, 7 * per + 3, 64 * per, 1 << 20):
        ws = torch.full((elems + 64,), 7.0, device="cuda")
        counts.add(api.tl_k_attention_cache8_plan(n, 1, heads, kv, d, elems)[1])
        check(api, c, n, k, v, q, heads, kv, ws[:elems])
        assert (ws[elems:] == 7.0).all()
    assert len(counts) >= 4


def test_scores_far_apart(api):
    """one key far above all others, early and late; scores of a thousand and below -1e4"""
    heads, d, n = 2, 64, 400
    k, v = draw(10, n, heads, d, big=1.0)
    for at in (0, 63, 64, 399):
        k2 = k.clone()
        k2[at] *= 100
        c = fill(api, k2, v, heads)
        for s in (1.0, -30.0):
            q = (k2[at:at + 1].float() * s / 8).bfloat16()
            check(api, c, n, k2, v, q, heads, heads)


def test_scales_far_apart(api):
    """blocks whose values, and whose keys, differ by many orders of magnitude"""
    heads, d, n = 1, 128, 330
    k, v = draw(11, n, heads, d)
    for j, f in enumerate((1e-30, 1.0, 1e30, 1e-5, 1e10)):
        v[j * 64:(j + 1) * 64] = (v[j * 64:(j + 1) * 64].float() * f).bfloat16()
        k[j * 64:(j + 1) * 64] = (k[j * 64:(j + 1) * 64].float() * (1e-20, 1e-3, 1e-2, 1.0, 0.1)[j]).bfloat16()
    c = fill(api, k, v, heads)
    check(api, c, n, k, v, queries(3, 1, d), heads, heads)
    check(api, c, n, k, v, queries(4, 40, d), heads, heads)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("rows", [1, 12, 20, 150])
@pytest.mark.parametrize("where", ["values", "keys"])
def test_values_that_are_not_finite(api, bad, rows, where):
    """rows that see them get what the formula gives; those that do not, and other heads, are as without them"""
    heads, d, n = 2, 64, 400
    k, v = draw(12, n, heads, d, big=1.0)
    q = queries(5, rows, heads * d)
    clean = attend(api, fill(api, k, v, heads), n, q, heads).view(rows, heads, d)
    x = v if where == "values" else k
    x[270, 3] = bad            # head 0, a complete block: that block, for every row that sees any of it
    x[395, d + 9] = bad        # head 1, the tail: rows that see token 395
    got = attend(api, fill(api, k, v, heads), n, q, heads).view(rows, heads, d)
    sees_block = torch.arange(rows) + n - rows >= 256
    sees_token = torch.arange(rows) + n - rows >= 395
    assert torch.isnan(got[sees_block, 0]).all()
    assert torch.equal(got[~sees_block, 0], clean[~sees_block, 0])
    assert torch.equal(got[~sees_token, 1], clean[~sees_token, 1])
    if where == "values":
        k, v = draw(12, n, heads, d, big=1.0)
        want, size, reach = oracle.attention(q, oracle.held(k, heads)[0], oracle.held(v, heads)[0], heads)
        far = (got.double() - want).abs() - oracle.attention_bound(want, size, reach, d, n, BF16)
        assert far[:, 1, [e for e in range(d) if e != 9]].max() <= 0
        assert torch.isnan(got[sees_token, 1, 9]).all() if math.isnan(bad) else (got[sees_token, 1, 9] == bad).all()
    elif math.isnan(bad):
        assert torch.isnan(got[sees_token, 1]).all()


def test_query_and_output_rows_of_other_strides(api):
    heads, kv, d, n = 4, 2, 64, 300
    k, v = draw(13, n, kv, d)
    c = fill(api, k, v, kv)
    for rows in (1, 7, 90):
        q = queries(6, rows, heads * d)
        want = attend(api, c, n, q, heads)
        for off in (0, 1, 3):
            qb = torch.full((rows * 300 + 8,), math.nan, dtype=torch.bfloat16, device="cuda")
            ob = torch.full((rows * 400 + 8,), 5.0, dtype=torch.bfloat16, device="cuda")
            qq, oo = qb[off:off + rows * 300].view(rows, 300)[:, 10:10 + heads * d], ob[off:off + rows * 400].view(rows, 400)[:, 20:20 + heads * d]
            qq.copy_(q)
            api.tl_k_attention_cache8(c, n, qq, oo, heads)
            assert torch.equal(oo.cpu(), want)
            oo.fill_(5.0)
            assert (ob == 5.0).all()


def test_nothing_to_do(api):
    c = api.Cache8.empty(2, 64, 100)
    e = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda")
    api.tl_k_cache8_append(c, 100, e, e)
    api.tl_k_attention_cache8(c, 50, e, e, 2)
    f = torch.empty(0, 128, device="cuda")
    api.tl_k_cache8_read(c, 100, 100, f, f)


def test_results_do_not_vary(api):
    heads, kv, d, n = 32, 8, 128, 3000
    k, v = draw(14, n, kv, d)
    c = fill(api, k, v, kv)
    ws = torch.empty(1 << 22, device="cuda")
    for rows in (1, 9, 300):
        q = queries(7, rows, heads * d)
        first = attend(api, c, n, q, heads, ws)
        for _ in range(4):
            assert torch.equal(first, attend(api, c, n, q, heads, ws))


def test_captured_steps(api):
    """append and attention of a few tokens as a graph, replayed behind a changed cache, beside eager work"""
    heads, d, n = 4, 64, 190
    k, v = draw(15, n + 8, heads, d)
    kd, vd = k.cuda(), v.cuda()
    q = queries(8, 1, heads * d).cuda()
    c = fill(api, k[:n], v[:n], heads, capacity=n + 8)
    start = {name: t.clone() for name, t in c.tensors.items()}
    ws = torch.empty(1 << 18, device="cuda")

    def steps(out):
        for i in range(8):         # token 191 completes a block
            api.tl_k_cache8_append(c, n + i, kd[n + i:n + i + 1], vd[n + i:n + i + 1])
            api.tl_k_attention_cache8(c, n + i + 1, q, out[i:i + 1], heads, ws)

    eager = torch.empty(8, heads * d, dtype=torch.bfloat16, device="cuda")
    steps(eager)
    out = torch.empty_like(eager)
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
        steps(out)
    torch.cuda.current_stream().wait_stream(s)
    for _ in range(3):
        for name, t in c.tensors.items():
            t.copy_(start[name])
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        torch.mm(torch.randn(64, 64, device="cuda"), torch.randn(64, 64, device="cuda"))


@pytest.mark.parametrize("rows", [1, 40])
def test_offsets_beyond_32_bits(api, rows):
    """2^31 bytes of codes and more lie before the last blocks"""
    heads, d, n = 32, 128, (1 << 19) + 200
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("24 GB of device memory needed")
    c = api.Cache8.empty(heads, d, n)
    g = torch.Generator(device="cuda").manual_seed(3)
    for name, t in c.tensors.items():
        if t.dtype == torch.int8:
            t.random_(-127, 128, generator=g)
        elif t.dtype == torch.float32:
            t.fill_(0.01)
    first = (1 << 19) - 64         # the last tokens come through append, over the 2^31-byte mark
    k, v = draw(21, n - first, heads, d)
    api.tl_k_cache8_append(c, first, k.cuda(), v.cuda())
    for x, got in zip((k, v), read(api, c, n, first, n - first)):
        assert same(got.view(-1, heads, d), oracle.held(x, heads)[0])
    q = queries(9, rows, heads * d) * 0.3
    q = q.bfloat16()
    o = torch.full((rows, heads * d), math.nan, dtype=torch.bfloat16, device="cuda")
    api.tl_k_attention_cache8(c, n, q.cuda(), o, heads, torch.empty(1 << 22, device="cuda"))
    full = n // 64
    for h in (0, 31):
        kh = (c.tensors["k"][:full, h].double() * c.tensors["k_scale"][:full, h].double()[:, None, None, None]).transpose(1, 2).reshape(-1, d)
        vh = (c.tensors["v"][:full, h].double() * c.tensors["v_scale"][:full, h].double()[:, None, None]).transpose(1, 2).reshape(-1, d)
        kh = torch.cat([kh, k[-(n - 64 * full):].view(-1, heads, d)[:, h].double().cuda()])
        vh = torch.cat([vh, v[-(n - 64 * full):].view(-1, heads, d)[:, h].double().cuda()])
        for i in {0, rows - 1}:
            see = n - rows + i + 1
            qi = q[i].view(heads, d)[h].double().cuda()
            p = torch.softmax(kh[:see] @ qi / math.sqrt(d), 0)
            want, size = p @ vh[:see], p @ vh[:see].abs()
            reach = (kh[:see].abs() @ qi.abs()).max() / math.sqrt(d)
            far = (o[i].view(heads, d)[h].double() - want).abs() - oracle.attention_bound(want, size, reach, d, n, BF16)
            assert far.max() <= 0, (h, i, far.max())


def test_two_streams_at_once(api):
    """calls on two streams, each with its cache and workspace, and a stream given by its handle"""
    heads, d, n = 8, 128, 2000
    sets = []
    for i in range(2):
        k, v = draw(30 + i, n, heads, d)
        q1, q2 = queries(31 + i, 1, heads * d).cuda(), queries(33 + i, 100, heads * d).cuda()
        c = fill(api, k, v, heads)
        ws = torch.empty(1 << 21, device="cuda")
        want = []
        for q in (q1, q2):
            o = torch.empty_like(q)
            api.tl_k_attention_cache8(c, n, q, o, heads, ws)
            want.append(o)
        sets.append((c, q1, q2, ws, want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        got = [(torch.empty_like(q1), torch.empty_like(q2)) for _, q1, q2, *_ in sets]
        torch.cuda.synchronize()
        for (c, q1, q2, ws, _, s), (o1, o2) in zip(sets, got):
            api.tl_k_attention_cache8(c, n, q1, o1, heads, ws, stream=s.cuda_stream)
            api.tl_k_attention_cache8(c, n, q2, o2, heads, ws, stream=s.cuda_stream)
        torch.cuda.synchronize()
        for (_, _, _, _, want, _), (o1, o2) in zip(sets, got):
            assert torch.equal(o1, want[0]) and torch.equal(o2, want[1])


@pytest.mark.parametrize("rows,heads,kv", [(1, 4, 4), (30, 4, 2), (300, 16, 16)])
def test_captured_attention(api, rows, heads, kv):
    """each kind of kernel, in a graph that is replayed between eager work on the same buffers"""
    d, n = 64, 1000
    k, v = draw(40, n, kv, d)
    c = fill(api, k, v, kv)
    q = queries(10, rows, heads * d).cuda()
    o, ws = torch.empty_like(q), torch.empty(1 << 21, device="cuda")
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    api.tl_k_attention_cache8(c, n, q, o, heads, ws)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
        api.tl_k_attention_cache8(c, n, q, o, heads, ws)
    torch.cuda.current_stream().wait_stream(s)
    for i in range(3):
        q.copy_(queries(11 + i, rows, heads * d))
        api.tl_k_attention_cache8(c, n, q, o, heads, ws)
        want = o.clone()
        o.zero_(), ws.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)


def test_rows_behind_the_last_are_left_alone(api):
    heads, d, n = 2, 64, 130
    k, v = draw(41, n, heads, d)
    c = fill(api, k, v, heads, capacity=300)
    before = {name: t.clone() for name, t in c.tensors.items()}
    api.tl_k_attention_cache8(c, n, queries(12, 5, heads * d).cuda(), torch.empty(5, heads * d, dtype=torch.bfloat16, device="cuda"), heads)
    for name, t in c.tensors.items():
        assert torch.equal(t.view(torch.uint8), before[name].view(torch.uint8)), name
    x, y = draw(42, 3, heads, d)
    api.tl_k_cache8_append(c, n, x.cuda(), y.cuda())
    for name in ("k", "v", "k_scale", "v_scale"):          # no block was completed
        assert torch.equal(c.tensors[name].view(torch.uint8), before[name].view(torch.uint8)), name
    kt = c.tensors["k_tail"].view(torch.int16)
    assert torch.equal(kt[:, :, 5:], before["k_tail"].view(torch.int16)[:, :, 5:]) and torch.equal(kt[:, :, :2], before["k_tail"].view(torch.int16)[:, :, :2])


def test_values_that_are_not_finite_in_wide_workgroups(api):
    n, rows, heads, _, d = WIDE[0]
    assert api.tl_k_attention_cache8_plan(n, rows, heads, heads, d)[0] == "rows256"
    k, v = draw(50, n, heads, d, big=1.0)
    q = queries(51, rows, heads * d)
    clean = attend(api, fill(api, k, v, heads), n, q, heads).view(rows, heads, d)
    v[590, 9] = math.inf               # head 0, the tail (tokens 576 ..)
    v[300, d + 3] = math.nan           # head 1, block 4
    got = attend(api, fill(api, k, v, heads), n, q, heads).view(rows, heads, d)
    at = torch.arange(rows) + n - rows
    assert torch.equal(got[:, 2:], clean[:, 2:])
    assert torch.isnan(got[at >= 256, 1]).all() and torch.equal(got[at < 256, 1], clean[at < 256, 1])
    assert (got[at >= 590, 0, 9] == math.inf).all()
    assert torch.equal(got[at < 576, 0], clean[at < 576, 0])
    rest = [e for e in range(d) if e != 9]
    # the same probabilities, as rounded, times the same values, summed in another order, and rounded to bf16: half a step of either
    size = v.view(n, heads, d)[:576, 0].float().abs().max()
    far = (got[:, 0].float() - clean[:, 0].float()).abs()
    bound = 2.0 ** -7 * clean[:, 0].float().abs() + 600 * 2.0 ** -23 * size
    assert (far[:, rest] <= bound[:, rest]).all() and (far[at < 590] <= bound[at < 590]).all()


@pytest.mark.parametrize("rows,heads,kv,n", [(1, 2, 2, 300), (1, 4, 2, 900), (12, 4, 4, 2000), (5, 6, 2, 130), (150, 2, 2, 400), (520, 64, 64, 600)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_query_that_is_not_finite(api, rows, heads, kv, n, bad):
    """is its own row and head's alone"""
    d = 64
    k, v = draw(60, n, kv, d)
    c = fill(api, k, v, kv)
    q = queries(61, rows, heads * d)
    ws = torch.full((1 << 20,), math.nan, device="cuda")
    clean = attend(api, c, n, q, heads, ws).view(rows, heads, d)
    hit = torch.zeros(rows, heads, dtype=torch.bool)
    for r, h in ((0, 0), (rows // 2, heads - 1), (rows - 1, heads // 2)):
        q[r, h * d + 7] = bad
        hit[r, h] = True
    got = attend(api, c, n, q, heads, ws).view(rows, heads, d)
    assert torch.equal(got[~hit], clean[~hit])
    assert torch.isnan(got[hit]).all()             # infinities among its scores: above all others, of either sign, or times a zero code


@pytest.mark.parametrize("n", [64, 128, 192, 193, 199])
def test_fewer_keys_than_are_cached(api, n):
    """a multiple of 64, or inside the tail"""
    heads, d = 2, 64
    k, v = draw(70, 200, heads, d)
    c = fill(api, k, v, heads)
    for rows in (1, 40):
        check(api, c, n, k, v, queries(rows, rows, heads * d), heads, heads)
    got = read(api, c, n, 1, n - 1)
    for x, y in zip((k, v), got):
        assert same(y.view(n - 1, heads, d), oracle.held(x, heads)[0][1:n])
