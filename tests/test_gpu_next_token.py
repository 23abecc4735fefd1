"""A step that has no token to choose: all logits undefined, or none allowed.  It returns TL_ERR_ARG whatever is set of penalties, bias and mask,
writes no output, and a decode step can be made again."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2401_11504_amd import synth  # noqa: E402
from test_gpu_kernels import H, api  # noqa: E402,F401

ARG = -1


def calls(api, lora, vocab):
    """the three steps as raw calls: (status, next_token, logits) with both outputs marked beforehand"""
    def call(f, *args):
        nxt, logits = C.c_int32(-77), np.full(vocab, 123.0, np.float32)
        st = f(lora, *args, C.byref(nxt), logits.ctypes.data)
        return st, nxt.value, logits

    def tokens(t):
        a = np.ascontiguousarray(t, np.int32)
        return a.ctypes.data, a.size, a

    def prefill(t):
        p, n, keep = tokens(t)
        return call(api._lib.tl_prefill, p, n)

    def extend(t):
        p, n, keep = tokens(t)
        return call(api._lib.tl_extend, p, n)

    return prefill, lambda t: call(api._lib.tl_decode_step, int(t)), extend


def refused_without_output(r):
    st, nxt, logits = r
    return st == ARG and nxt == -77 and (logits == 123.0).all()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("penalties", [False, True])
@pytest.mark.parametrize("n", [20, 63])
def test_undefined_logits(api, H, eight, penalties, n):
    shape = synth.SHAPES["small"]
    V = shape.vocab
    model = H.Model(shape, 6100, max_tokens=100)
    (a, _), (b, _) = (H.new_lora(model, 6100, b_std=0.01) for _ in range(2))
    text = synth.zipf_tokens(6100, 100, V)
    good = api.tl_get_factor(a, 0, 6, api.FACTOR_B, (shape.d_model, shape.rank))
    bad = good.copy()
    bad[5, 3] = np.nan         # the first layer's down projection: one element of the residual stream, so the next layer's keys and values and all logits
    for m in (a, b):
        api.tl_cache_8bit(m, eight)
        if penalties:
            api.tl_set_penalties(m, 1.2, 0.1, 0.1)
        api.tl_prefill(m, text[:n])
    prefill, step, extend = calls(api, a, V)
    api.tl_set_factor(a, 0, 6, api.FACTOR_B, bad)
    assert refused_without_output(step(text[n]))
    assert api.tl_kv_length(a) == n
    api.tl_set_factor(a, 0, 6, api.FACTOR_B, good)
    for i in range(n, n + 3):                                    # the step again, and on
        xa, xb = api.tl_decode_step(a, text[i], V), api.tl_decode_step(b, text[i], V)
        assert xa[0] == xb[0] and np.array_equal(xa[1], xb[1])
    api.tl_set_factor(a, 0, 6, api.FACTOR_B, bad)
    if eight:
        assert refused_without_output(extend(text[n + 3:n + 9]))
        assert api.tl_kv_length(a) == 0
    assert refused_without_output(prefill(text[:n]))
    assert api.tl_kv_length(a) == 0
    with pytest.raises(api.TlError) as e:
        api.tl_generate(a, text[:n], 4, 30, 10, n_ctx_max=40)
    assert e.value.status == ARG
    api.tl_set_factor(a, 0, 6, api.FACTOR_B, good)
    assert prefill(text[:n])[0] == 0
    for m in (a, b):
        api.tl_lora_free(m)
    model.close()


def test_no_token_allowed_writes_nothing(api, H):
    shape = synth.SHAPES["small"]
    V = shape.vocab
    model = H.Model(shape, 6200, max_tokens=100)
    a, _ = H.new_lora(model, 6200, b_std=0.01)
    text = synth.zipf_tokens(6200, 100, V)
    api.tl_cache_8bit(a, True)
    prefill, step, extend = calls(api, a, V)
    assert prefill(text[:30])[0] == 0
    api.tl_set_allowed(a, np.zeros(V, bool), V)
    assert refused_without_output(step(text[30])) and api.tl_kv_length(a) == 30
    assert refused_without_output(extend(text[30:40]))
    assert refused_without_output(prefill(text[:30]))
    api.tl_lora_free(a)
    model.close()
