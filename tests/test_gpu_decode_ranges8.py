"""Decoding over the 8-bit cache where a row's keys are cut into ranges, and each of the attention's kernels in a captured graph.  Which kernel and how
many ranges the sizes get is asserted, so that no path is left untested when the rule changes."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2401_11504_amd import synth  # noqa: E402
from test_gpu_cache8 import draw, fill, queries  # noqa: E402
from test_gpu_generate8 import close, logits_given_kv, make  # noqa: E402
from test_gpu_kernels import BF16_TOL, H, api, check  # noqa: E402,F401

WORKSPACE = 1 << 22    # floats, the module's own


@pytest.mark.parametrize("name,n,kernel,ranges", [
    ("small", 701, "columns8", (1, 1, 1, 4, 4)),       # kept in one up to 704 keys (eight waves a workgroup), cut behind
    ("small", 766, "columns16", (4, 4, 5, 5, 5)),      # and over the step that completes a block
    ("small", 1500, "columns16", (8,) * 5), ("small128", 1500, "columns16", (8,) * 5),
    ("small", 4094, "columns8", (16, 16, 22, 22, 22)), ("small128", 4094, "columns8", (16, 16, 22, 22, 22))])
def test_decode_over_ranges(api, H, name, n, kernel, ranges):
    shape = synth.SHAPES[name]
    model, (a,), facs = make(H, shape, 6800, n + 8, n=1)
    text = synth.zipf_tokens(6800, n + 8, shape.vocab)
    api.tl_cache_8bit(a, True)
    api.tl_prefill(a, text[:n])
    plans = []
    for i in range(n, n + 5):
        plans.append(api.tl_k_attention_cache8_plan(i + 1, 1, shape.n_heads, shape.n_heads, shape.d_head, WORKSPACE)[:2])
        nxt, logits = api.tl_decode_step(a, text[i], shape.vocab)
        assert nxt == int(np.argmax(logits))
        check(logits, logits_given_kv(api, a, model, shape, facs, text[i:i + 1]), BF16_TOL, f"logits behind {i + 1} tokens")
    close(api, model, a)
    assert tuple(p[1] for p in plans) == ranges and kernel in {p[0] for p in plans}, plans


CAPTURED = [("columns8", 1, 4, 4, 5000), ("columns8", 5, 16, 16, 400), ("columns16", 1, 4, 4, 1000), ("columns16", 12, 4, 4, 2000),
            ("rows128", 30, 4, 2, 1000), ("rows256", 520, 64, 64, 600)]


def test_all_kernels_are_captured():
    assert {c[0] for c in CAPTURED} == {"columns8", "columns16", "rows128", "rows256"}


@pytest.mark.parametrize("kernel,rows,heads,kv,n", CAPTURED)
def test_captured(api, kernel, rows, heads, kv, n):
    """replayed between eager calls on the same buffers"""
    d = 64
    k, v = draw(90, n, kv, d)
    c = fill(api, k, v, kv)
    q = queries(91, rows, heads * d).cuda()
    o, ws = torch.empty_like(q), torch.empty(WORKSPACE, device="cuda")
    assert api.tl_k_attention_cache8_plan(n, rows, heads, kv, d, WORKSPACE)[0] == kernel
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    api.tl_k_attention_cache8(c, n, q, o, heads, ws)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
        api.tl_k_attention_cache8(c, n, q, o, heads, ws)
    torch.cuda.current_stream().wait_stream(s)
    for i in range(4):
        q.copy_(queries(92 + i, rows, heads * d))
        api.tl_k_attention_cache8(c, n, q, o, heads, ws)
        want = o.clone()
        o.zero_(), ws.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
