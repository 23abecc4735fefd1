"""Generation over the 8-bit cache and the choice of the next token, through the module's own calls: what the cache holds against the
definition applied to the bf16 cache of a twin, logits against the oracle's layers over the keys and values that the cache stands for, the
choice against its definition."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import templora_oracle as O  # noqa: E402
from paper_2401_11504_amd import synth  # noqa: E402
from test_gpu_kernels import BF16_TOL, H, api, check  # noqa: E402,F401
import cache8_oracle  # noqa: E402

F64 = np.float64


def make(H, shape, seed, max_tokens, n=2, **kw):
    model = H.Model(shape, seed, max_tokens=max_tokens)
    mods = [H.new_lora(model, seed, b_std=0.01, **kw) for _ in range(n)]
    return model, [m[0] for m in mods], mods[0][1]


def close(api, model, *mods):
    for m in mods:
        api.tl_lora_free(m)
    model.close()


def kv(api, lora, shape, layer):
    return api.tl_get_kv(lora, layer, 0, api.tl_kv_length(lora), shape.d_model)


def held(x, shape):
    return cache8_oracle.held(torch.from_numpy(x).bfloat16(), shape.n_heads)[0].numpy().reshape(x.shape)


def logits_given_kv(api, lora, model, shape, facs, tokens):
    """The last position's logits: the tokens (the last ones of the cached text) go through the layers in fp64, every layer's attention over the
    keys and values that the cache stands for (tl_get_kv), causal."""
    nh, dh, s = shape.n_heads, shape.d_head, shape.scale
    n, T = api.tl_kv_length(lora), len(tokens)
    h = np.asarray(model.emb, F64)[np.asarray(tokens)]
    fresh = []
    for l in range(shape.n_layers):
        W, L = model.host_layers[l], facs[l]
        K, V = (x.astype(F64).reshape(n, nh, dh) for x in kv(api, lora, shape, l))
        x1 = O.rmsnorm_fwd(h, W["g1"], shape.rms_eps)
        q, k = (O.rope_fwd(O.lora_linear_fwd(x1, W[p], *L[p], s)[0].reshape(T, nh, dh), shape.rope_base, n - T) for p in "qk")
        fresh.append((k, O.lora_linear_fwd(x1, W["v"], *L["v"], s)[0].reshape(T, nh, dh), K[n - T:], V[n - T:]))
        o = np.zeros((T, nh, dh))
        for i in range(T):
            see = n - T + i + 1
            sc = np.einsum("hd,uhd->hu", q[i], K[:see]) / np.sqrt(dh)
            sc = np.exp(sc - sc.max(1, keepdims=True))
            o[i] = np.einsum("hu,uhd->hd", sc / sc.sum(1, keepdims=True), V[:see])
        h1 = h + O.lora_linear_fwd(o.reshape(T, nh * dh), W["o"], *L["o"], s)[0]
        x2 = O.rmsnorm_fwd(h1, W["g2"], shape.rms_eps)
        a = O.swiglu_fwd(O.lora_linear_fwd(x2, W["gate"], *L["gate"], s)[0], O.lora_linear_fwd(x2, W["up"], *L["up"], s)[0])
        h = h1 + O.lora_linear_fwd(a, W["down"], *L["down"], s)[0]
    # what the cache holds of the new tokens is what they give, within bf16 and half a code (127 codes to the largest magnitude of a block)
    for l, (k, v, K, V) in enumerate(fresh):
        for got, want in ((K, k), (V, v)):
            rms = np.sqrt(np.mean(want * want))
            # (a block's largest magnitude may lie before these tokens: five standard deviations cover 64 x 128 normal draws four times in five, seven all)
            assert np.linalg.norm(got - want) / np.linalg.norm(want) <= BF16_TOL + max(np.abs(want).max() / rms, 7.0) / 254, l
    return (O.rmsnorm_fwd(h, np.ones(shape.d_model), shape.rms_eps) @ np.asarray(model.head, F64).T)[-1]


# ---------------------------------------------------------------- what the cache holds
@pytest.mark.parametrize("name", ["small", "small128"])
@pytest.mark.parametrize("n", [1, 50, 64, 130])
def test_prefill_and_decode_fill_the_cache(api, H, name, n):
    shape = synth.SHAPES[name]
    model, (a, b), _ = make(H, shape, 5100, n + 70)
    text = synth.zipf_tokens(5100, n + 70, shape.vocab)
    api.tl_cache_8bit(a, True)
    na, la = api.tl_prefill(a, text[:n], shape.vocab)
    nb, lb = api.tl_prefill(b, text[:n], shape.vocab)
    assert na == nb and np.array_equal(la, lb)                   # the prompt's own attention is the same
    for l in range(shape.n_layers):
        for x, y in zip(kv(api, a, shape, l), kv(api, b, shape, l)):
            assert np.array_equal(x, held(y, shape))
    for i in range(n, n + 70):                                   # over a border of two blocks
        api.tl_decode_step(a, text[i])
        api.tl_decode_step(b, text[i])
        if i % 16 == 0 or i % 64 in (0, 62, 63) or i == n + 69:  # the first layer's keys and values depend on the tokens alone
            for x, y in zip(kv(api, a, shape, 0), kv(api, b, shape, 0)):
                assert np.array_equal(x, held(y, shape)), i
    close(api, model, a, b)


@pytest.mark.parametrize("name", ["small", "small128"])
def test_decode_logits(api, H, name):
    shape = synth.SHAPES[name]
    model, (a,), facs = make(H, shape, 5200, 700, n=1)
    text = synth.zipf_tokens(5200, 700, shape.vocab)
    api.tl_cache_8bit(a, True)
    for n in (1, 61, 127, 600):                                  # 600: the keys are cut into ranges
        api.tl_prefill(a, text[:n])
        for i in range(n, n + 5):
            nxt, logits = api.tl_decode_step(a, text[i], shape.vocab)
            assert nxt == int(np.argmax(logits))
            check(logits, logits_given_kv(api, a, model, shape, facs, text[i:i + 1]), BF16_TOL, f"logits behind {i + 1} tokens")
    close(api, model, a)


@pytest.mark.parametrize("name", ["small", "small128"])
@pytest.mark.parametrize("n,T", [(1, 1), (40, 7), (60, 70), (128, 64), (200, 333)])
def test_extend(api, H, name, n, T):
    shape = synth.SHAPES[name]
    model, (a, b), facs = make(H, shape, 5300, n + T + 3)
    text = synth.zipf_tokens(5300, n + T + 3, shape.vocab)
    for m in (a, b):
        api.tl_cache_8bit(m, True)
        api.tl_prefill(m, text[:n])
    nxt, logits = api.tl_extend(a, text[n:n + T], shape.vocab)
    assert api.tl_kv_length(a) == n + T and nxt == int(np.argmax(logits))
    check(logits, logits_given_kv(api, a, model, shape, facs, text[n:n + T]), BF16_TOL, "logits")
    for t in text[n:n + T]:
        _, lb = api.tl_decode_step(b, t, shape.vocab)
    for x, y in zip(kv(api, a, shape, 0), kv(api, b, shape, 0)): # the same tokens: bf16 roundings of differently ordered sums, and half a code
        assert np.linalg.norm(x - y) <= (BF16_TOL + 7 / 254) * np.linalg.norm(y)
    # the text goes on from it
    for i in range(n + T, n + T + 3):
        _, logits = api.tl_decode_step(a, text[i], shape.vocab)
        check(logits, logits_given_kv(api, a, model, shape, facs, text[i:i + 1]), BF16_TOL, "logits after extend")
    close(api, model, a, b)


def test_switching_and_reuse(api, H):
    shape = synth.SHAPES["small"]
    model, (a, b), _ = make(H, shape, 5400, 120)
    text = synth.zipf_tokens(5400, 120, shape.vocab)
    api.tl_cache_8bit(a, True)
    api.tl_prefill(a, text[:80])
    api.tl_prefill(b, text[:80])
    api.tl_cache_8bit(b, True)                                   # the cache moves along
    api.tl_cache_8bit(b, True)
    assert api.tl_kv_length(b) == 80
    for i in range(80, 84):
        xa, xb = api.tl_decode_step(a, text[i], shape.vocab), api.tl_decode_step(b, text[i], shape.vocab)
        assert xa[0] == xb[0] and np.array_equal(xa[1], xb[1])
    # a training call drops it, unless it is to be kept
    api.tl_chunk_loss(a, text[:32])
    assert api.tl_kv_length(a) == 0
    with pytest.raises(api.TlError) as e:
        api.tl_extend(a, text[:3])
    assert e.value.status == -1
    api.tl_cache_reuse(b, True)
    before = kv(api, b, shape, 1)
    api.tl_chunk_update(b, text[:32], 0, 1e-3)
    assert api.tl_kv_length(b) == 84
    for x, y in zip(before, kv(api, b, shape, 1)):
        assert np.array_equal(x, y)
    nxt, _ = api.tl_decode_step(b, text[84])
    api.tl_extend(b, text[85:110])
    # back to bf16: dropped, and the same as a module that never had it
    api.tl_cache_8bit(b, False)
    assert api.tl_kv_length(b) == 0
    api.tl_cache_reuse(a, True)                                  # with the 8-bit cache on ..
    api.tl_cache_8bit(a, False)                                  # .. and then off: the bf16 buffers are there
    api.tl_set_factor(b, 0, 0, api.FACTOR_A, api.tl_get_factor(b, 0, 0, api.FACTOR_A, (shape.rank, shape.d_model)))
    c, _ = H.new_lora(model, 5400, b_std=0.01)
    for m in (a, c):
        api.tl_prefill(m, text[:40])
    for i in range(40, 44):
        xa, xc = api.tl_decode_step(a, text[i], shape.vocab), api.tl_decode_step(c, text[i], shape.vocab)
        assert xa[0] == xc[0] and np.array_equal(xa[1], xc[1])
    assert nxt >= 0
    close(api, model, a, b, c)


def test_two_modules_on_one_model(api, H):
    """each has its cache and its choice"""
    shape = synth.SHAPES["small"]
    model, (a, b), _ = make(H, shape, 5450, 100)
    text = synth.zipf_tokens(5450, 100, shape.vocab)
    for m in (a, b):
        api.tl_cache_8bit(m, True)
    api.tl_set_penalties(b, 1.5, 0.5, 0.1)
    alone = []
    for i in range(60, 70):
        if i == 60:
            api.tl_prefill(a, text[:60])
        alone.append(api.tl_decode_step(a, text[i], shape.vocab))
    api.tl_prefill(a, text[:60])
    api.tl_prefill(b, text[10:70])
    for i in range(60, 70):
        x = api.tl_decode_step(a, text[i], shape.vocab)
        api.tl_decode_step(b, text[i])
        assert x[0] == alone[i - 60][0] and np.array_equal(x[1], alone[i - 60][1])
    close(api, model, a, b)


# ---------------------------------------------------------------- the choice
def best(logits, text, vocab, rep=1.0, pres=0.0, freq=0.0, last_n=0, bias=None, allowed=None):
    """(index, values in fp64): of values rounded to fp32 step by step"""
    f = np.float32
    x = logits.astype(f)
    t = text[-last_n:] if last_n else text
    c = np.bincount(np.asarray(t, np.int64), minlength=vocab)
    with np.errstate(all="ignore"):
        y = np.where(x > 0, x / f(rep), x * f(rep)) - (f(freq) * c.astype(f) + f(pres))
    x = np.where(c > 0, y, x).astype(f)
    if bias is not None:
        x = x + bias.astype(f)
    if allowed is not None:
        x = np.where(allowed, x, -np.inf)
    return int(np.argmax(x))


@pytest.mark.parametrize("eight", [False, True])
def test_penalties_bias_and_mask(api, H, eight):
    shape = synth.SHAPES["small"]
    V = shape.vocab
    model, (a,), _ = make(H, shape, 5500, 300, n=1)
    g = np.random.default_rng(5)
    text = [int(t) for t in synth.zipf_tokens(5500, 150, V)]
    api.tl_cache_8bit(a, eight)
    bias = (g.normal(size=V) * (g.random(V) < 0.2)).astype(np.float32)
    allowed = g.random(V) < 0.6
    for kw, bi, al in ((dict(rep=1.5), None, None), (dict(rep=1.3, pres=0.4, freq=0.2, last_n=17), None, None), (dict(), bias, None),
                       (dict(), None, allowed), (dict(rep=0.7, pres=-0.3, freq=0.05), bias, allowed), (dict(), None, None)):
        api.tl_set_penalties(a, kw.get("rep", 1.0), kw.get("pres", 0.0), kw.get("freq", 0.0), kw.get("last_n", 0))
        api.tl_set_bias(a, bi, V)
        api.tl_set_allowed(a, al, V)
        seq = list(text[:100])
        nxt, logits = api.tl_prefill(a, seq, V)
        assert nxt == best(logits, seq, V, bias=bi, allowed=al, **kw)
        for _ in range(6):
            seq.append(nxt)
            nxt, logits = api.tl_decode_step(a, nxt, V)
            assert nxt == best(logits, seq, V, bias=bi, allowed=al, **kw)
        if eight:
            seq += text[110:140]
            nxt, logits = api.tl_extend(a, text[110:140], V)
            assert nxt == best(logits, seq, V, bias=bi, allowed=al, **kw)
    close(api, model, a)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n", [20, 63, 64])
def test_no_token_allowed_and_again(api, H, eight, n):
    shape = synth.SHAPES["small"]
    V = shape.vocab
    model, (a, b), _ = make(H, shape, 5600, 80)
    text = synth.zipf_tokens(5600, 80, V)
    for m in (a, b):
        api.tl_cache_8bit(m, eight)
        api.tl_prefill(m, text[:n])
    one = np.zeros(V, bool)
    api.tl_set_allowed(a, one, V)
    with pytest.raises(api.TlError) as e:
        api.tl_decode_step(a, text[n])
    assert e.value.status == -1 and api.tl_kv_length(a) == n
    one[7] = True
    api.tl_set_allowed(a, one, V)
    nxt, la = api.tl_decode_step(a, text[n], V)
    _, lb = api.tl_decode_step(b, text[n], V)
    assert nxt == 7 and np.array_equal(la, lb)
    api.tl_set_allowed(a, None, V)
    for i in range(n + 1, n + 4):
        xa, xb = api.tl_decode_step(a, text[i], V), api.tl_decode_step(b, text[i], V)
        assert xa[0] == xb[0] and np.array_equal(xa[1], xb[1])
    api.tl_set_allowed(a, np.zeros(V, bool), V)
    with pytest.raises(api.TlError):
        api.tl_prefill(a, text[:9])
    assert api.tl_kv_length(a) == 0
    close(api, model, a, b)


def test_generate_with_all_of_it(api, H):
    """tl_generate over the 8-bit cache with penalties and a mask, training included, against the same loop of single calls"""
    shape = synth.SHAPES["small"]
    V, window, chunk = shape.vocab, 90, 50
    model, (a, b), _ = make(H, shape, 5700, window + chunk)
    prompt = [int(t) for t in synth.zipf_tokens(5700, 100, V)]
    allowed = np.ones(V, bool)
    allowed[::7] = False
    for m in (a, b):
        api.tl_cache_8bit(m, True)
        api.tl_set_penalties(m, 1.2, 0.1, 0.1, 64)
        api.tl_set_allowed(m, allowed, V)
    out, losses = api.tl_generate(a, prompt, 120, window, chunk, n_ctx_max=40, batch=25, epochs=2, lr=1e-3)
    text, want, want_loss = list(prompt), [], []
    while len(want) < 120:
        nxt, _ = api.tl_prefill(b, text[-window:])
        got = 0
        while got < chunk and len(want) < 120:
            text.append(nxt)
            want.append(nxt)
            got += 1
            if got < chunk and len(want) < 120:
                nxt, _ = api.tl_decode_step(b, nxt)
        if got < chunk:
            break
        want_loss += api.tl_chunk_train(b, text[-(40 + chunk):], chunk, 40, 25, 2, 1e-3)
    assert list(out) == want and list(losses) == want_loss
    assert not any(t % 7 == 0 for t in out)
    close(api, model, a, b)


# ---------------------------------------------------------------- refusals
def refused(api, status, f, *args):
    with pytest.raises(api.TlError) as e:
        f(*args)
    assert e.value.status == status, e.value


def test_refusals(api, H):
    shape = synth.SHAPES["small"]
    V = shape.vocab
    model, (a,), _ = make(H, shape, 5800, 40, n=1)
    text = synth.zipf_tokens(5800, 60, V)
    refused(api, -1, api.tl_extend, a, text[:3])                 # the cache is not in 8 bits
    api.tl_cache_8bit(a, True)
    refused(api, -1, api.tl_extend, a, text[:3])                 # and empty
    refused(api, -1, api.tl_decode_step, a, 1)
    refused(api, -4, api.tl_prefill, a, text[:41])
    refused(api, -4, api.tl_prefill, a, [])
    api.tl_prefill(a, text[:30])
    for t, status in ((text[:11], -4), ([], -4), ([1, V], -3), ([-1], -3)):
        refused(api, status, api.tl_extend, a, t)
    assert api.tl_kv_length(a) == 30                             # refused calls change nothing
    api.tl_extend(a, text[30:40])
    assert api.tl_kv_length(a) == 40
    refused(api, -4, api.tl_extend, a, text[:1])
    refused(api, -4, api.tl_decode_step, a, 1)
    for layer, first, n, status in ((-1, 0, 1, -1), (2, 0, 1, -1), (0, -1, 1, -4), (0, 0, -1, -4), (0, 40, 1, -4), (0, 2 ** 31 - 1, 2 ** 31 - 1, -4)):
        k = np.empty(4, np.float32)
        assert api._lib.tl_get_kv(a, layer, first, n, k.ctypes.data, k.ctypes.data) == status
    assert api._lib.tl_get_kv(a, 0, 0, 1, None, None) == -1
    nan = float("nan")
    for bad in ((0.0, 0, 0, 0), (-1.0, 0, 0, 0), (nan, 0, 0, 0), (1.0, nan, 0, 0), (1.0, 0, float("inf"), 0), (1.1, 0, 0, -1)):
        refused(api, -1, api.tl_set_penalties, a, *bad)
    api.tl_discard(a)
    for f, args in ((api.tl_cache_8bit, (a, True)), (api.tl_extend, (a, text[:1])), (api.tl_set_penalties, (a, 1.2)), (api.tl_set_bias, (a, None, V)),
                    (api.tl_set_allowed, (a, None, V)), (api.tl_get_kv, (a, 0, 0, 1, 4))):
        refused(api, -7, f, *args)
    close(api, model, a)
    for f, args in ((api.tl_cache_8bit, (None, True)), (api.tl_extend, (None, text[:1])), (api.tl_set_penalties, (None, 1.2))):
        refused(api, -1, f, *args)
    bare = H.Model(synth.SHAPES["layer"], 5800, max_tokens=8)    # no lm_head: nothing to choose from
    b, _ = H.new_lora(bare, 5800)
    for f, args in ((api.tl_set_penalties, (b, 1.2)), (api.tl_set_bias, (b, np.zeros(3), 3)), (api.tl_set_allowed, (b, [True], 1))):
        refused(api, -2, f, *args)
    close(api, bare, b)
