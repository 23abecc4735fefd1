"""The module's generation with drawn tokens: what tl_prefill, tl_decode_step, tl_extend and tl_generate draw is what the definition draws from
the logits they give back, behind penalties, bias and mask."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2401_11504_amd import synth  # noqa: E402
from test_gpu_kernels import H, api  # noqa: E402,F401
import paged_oracle as oracle  # noqa: E402

M64 = (1 << 64) - 1


def mix64(z):
    z = (z + 0x9E3779B97F4A7C15) & M64
    z = ((z ^ z >> 30) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ z >> 27) * 0x94D049BB133111EB) & M64
    return z ^ z >> 31


def number(seed, i):
    return (mix64((mix64(seed) + i) & M64) >> 40) * 2.0 ** -24


def want(logits, settings, seed, i):
    x = torch.from_numpy(np.asarray(logits, np.float32))[None]
    return oracle.sample(x, torch.tensor([settings], dtype=torch.float32), torch.tensor([number(seed, i)]))[0][0]


@pytest.fixture
def module(H, api):
    shape = synth.SHAPES["small"]
    model = H.Model(shape, 31, max_tokens=120)
    lora = H.new_lora(model, 31, b_std=0.01)[0]
    yield shape, lora
    api.tl_lora_free(lora)
    model.close()


@pytest.mark.parametrize("settings", [(1.0, 0, 1.0, 0.0), (0.8, 5, 0.9, 0.01), (5.0, 0, 0.7, 0.0), (3.0, 40, 1.0, 0.3), (0.0, 0, 1.0, 0.0)])
@pytest.mark.parametrize("seed", [0, 2 ** 63 + 5])
def test_steps_draw_by_the_definition(api, module, settings, seed):
    shape, lora = module
    T, k, p, m = settings
    api.tl_set_sampling(lora, T, k, p, m, seed)
    tok, logits = api.tl_prefill(lora, [3, 1, 4, 1, 5], shape.vocab)
    for i in range(8):
        assert tok == want(logits, settings, seed, i), i
        tok, logits = api.tl_decode_step(lora, tok, shape.vocab)
    api.tl_set_sampling(lora)                                  # greedy again
    tok, logits = api.tl_decode_step(lora, tok, shape.vocab)
    assert tok == int(np.argmax(logits))


def test_behind_penalties_bias_and_mask(api, module):
    shape, lora = module
    V, seed, settings = shape.vocab, 9, (2.0, 20, 0.95, 0.0)
    rng = np.random.RandomState(3)
    bias, allowed = rng.randn(V).astype(np.float32), rng.rand(V) < 0.3
    api.tl_set_penalties(lora, 1.3, 0.2, 0.1)
    api.tl_set_bias(lora, bias, V)
    api.tl_set_allowed(lora, allowed, V)
    api.tl_set_sampling(lora, 2.0, 20, 0.95, 0.0, seed)
    text = [3, 1, 4, 1, 5]
    tok, logits = api.tl_prefill(lora, text, V)
    for i in range(6):
        x = torch.from_numpy(logits)[None].cuda()
        counts = torch.bincount(torch.tensor(text), minlength=V).int()[None].cuda()
        bits = np.packbits(allowed, bitorder="little")
        words = np.zeros(4 * ((V + 31) // 32), np.uint8)
        words[:bits.size] = bits
        out = torch.empty_like(x)
        api.tl_k_choose(x, counts, out, None, 1.3, 0.2, 0.1, torch.from_numpy(bias)[None].cuda(), torch.from_numpy(words.view(np.int32).copy())[None].cuda())
        assert tok == want(out[0].cpu().numpy(), settings, seed, i) and allowed[tok]
        text.append(tok)
        tok, logits = api.tl_decode_step(lora, tok, V)


def test_generate_and_extend(api, module):
    shape, lora = module
    V = shape.vocab
    run = lambda seed: (api.tl_set_sampling(lora, 4.0, 0, 1.0, 0.0, seed),  # noqa: E731
                        api.tl_generate(lora, [1, 2, 3], 20, window=40, chunk=30, n_ctx_max=10)[0])[1].tolist()
    a, b, c = run(1), run(1), run(2)
    assert a == b and a != c and all(0 <= t < V for t in a)
    # the same as steps make them
    api.tl_set_sampling(lora, 4.0, 0, 1.0, 0.0, 1)
    tok, _ = api.tl_prefill(lora, [1, 2, 3])
    got = [tok]
    for _ in range(19):
        tok, _ = api.tl_decode_step(lora, tok)
        got.append(tok)
    assert got == a
    api.tl_cache_8bit(lora)
    api.tl_set_sampling(lora, 3.0, 0, 0.9, 0.0, 77)
    tok, logits = api.tl_prefill(lora, [1, 2, 3], V)
    assert tok == want(logits, (3.0, 0, 0.9, 0.0), 77, 0)
    tok, logits = api.tl_extend(lora, [5, 6, 7], V)
    assert tok == want(logits, (3.0, 0, 0.9, 0.0), 77, 1)


def test_refusals_and_steps_that_fail(api, module):
    shape, lora = module
    V = shape.vocab
    for bad in ((-1.0, 0, 1.0, 0.0), (math.nan, 0, 1.0, 0.0), (math.inf, 0, 1.0, 0.0), (1.0, -1, 1.0, 0.0), (1.0, 0, math.nan, 0.0), (1.0, 0, 1.0, math.inf)):
        with pytest.raises(api.TlError):
            api.tl_set_sampling(lora, *bad)
    api.tl_set_sampling(lora, 3.0, 0, 1.0, 0.0, 5)
    tok, logits = api.tl_prefill(lora, [1, 2, 3], V)
    assert tok == want(logits, (3.0, 0, 1.0, 0.0), 5, 0)
    n = api.tl_kv_length(lora)
    api.tl_set_allowed(lora, np.zeros(V, bool), V)
    with pytest.raises(api.TlError):
        api.tl_decode_step(lora, tok)
    assert api.tl_kv_length(lora) == n
    api.tl_set_allowed(lora, None, V)
    nxt, logits = api.tl_decode_step(lora, tok, V)             # made again; the one that failed drew nothing
    assert nxt == want(logits, (3.0, 0, 1.0, 0.0), 5, 1)
    api.tl_discard(lora)
    with pytest.raises(api.TlError) as e:
        api.tl_set_sampling(lora, 1.0)
    assert e.value.status == -7
