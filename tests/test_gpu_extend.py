"""tl_extend: no token of a call has part in what the tokens before it become.  Codes of a block share a scale, so a token that stands out takes the
others of its block down to coarse codes: the tokens before it must not have attended to those."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import cache8_oracle  # noqa: E402
from paper_2401_11504_amd import synth  # noqa: E402
from test_gpu_kernels import BF16_TOL, H, api  # noqa: E402,F401

LOUD = 7           # the token that stands out
CODE = 7 / 254     # half a code, with a block's largest magnitude at seven times its root mean square (64 x 64 normal draws stay below five)


def loud_model(api, H, shape, seed, max_tokens):
    """Token LOUD alone has a part in direction 0, which the first layer's value projection makes some thousand times as large as other values;
    nothing else reads direction 0.  Returns (handle, keep-alive list)."""
    def dev(x):
        return H.to_dev_bf16(x)
    ptrs = []
    for l in range(shape.n_layers):
        W = synth.layer_weights(seed, shape, l)
        for p in synth.PROJ:
            w = W[p].copy()
            if p in ("q", "k", "v", "gate", "up"):
                w[:, 0] = 100.0 if (p, l) == ("v", 0) else 0.0
            if p in ("o", "down"):
                w[0] = 0.0                             # and nothing else writes it
            ptrs.append(dev(w))
        ptrs += [torch.ones(shape.d_model, device="cuda") for _ in range(2)]
    emb, head = synth.embedding(seed, shape).copy(), synth.lm_head(seed, shape).copy()
    emb[:, 0] = 0.0
    emb[LOUD] = 0.0
    emb[LOUD, 0] = 0.5
    head[:, 0] = 0.0
    ptrs += [dev(emb), torch.ones(shape.d_model, device="cuda"), dev(head)]
    torch.cuda.synchronize()
    return api.tl_model_create(shape.n_layers, shape.d_model, shape.n_heads, shape.d_head, shape.d_ffn, shape.vocab, max_tokens, ptrs,
                               shape.rms_eps, shape.rope_base)


def module(api, model, shape, seed):
    """a module that leaves direction 0 alone"""
    lora = api.tl_lora_init(model, shape.rank, shape.alpha, seed=seed)
    for l in range(shape.n_layers):
        for i, (p, (a, b)) in enumerate(synth.lora_factors(seed, shape, l, b_std=0.01).items()):
            a, b = a.copy(), b.copy()
            if p in ("q", "k", "v", "gate", "up"):
                a[:, 0] = 0.0
            else:
                b[0] = 0.0
            api.tl_set_factor(lora, l, i, api.FACTOR_A, a)
            api.tl_set_factor(lora, l, i, api.FACTOR_B, b)
    return lora


def text_of(seed, n, vocab, loud):
    t = synth.zipf_tokens(seed, n, vocab)
    t[t == LOUD] = LOUD + 1
    t[loud] = LOUD
    return t


def kv(api, lora, shape, layer, first, n):
    return api.tl_get_kv(lora, layer, first, n, shape.d_model)


def held(x, shape):
    return cache8_oracle.held(torch.from_numpy(x).bfloat16(), shape.n_heads)[0].numpy().reshape(x.shape)


def far(x, y):
    return np.linalg.norm(x - y) / np.linalg.norm(y)


@pytest.mark.parametrize("name", ["small", "small128"])
@pytest.mark.parametrize("n,T,loud", [(5, 59, 62), (5, 70, 63), (40, 200, 127), (70, 58, 127), (130, 9, 135), (112, 16, 127), (60, 300, 188),
                                      (1530, 10, 1535), (4090, 8, 4095), (1500, 100, 1535)])
def test_a_later_token_of_the_block(api, H, name, n, T, loud):
    """against a twin that takes the same tokens step by step: the second layer's keys and values of the tokens before the loud one"""
    shape = synth.SHAPES[name]
    model = loud_model(api, H, shape, 6300, n + T)
    a, b = (module(api, model, shape, 6300) for _ in range(2))
    text = text_of(6300, n + T, shape.vocab, loud)
    for m in (a, b):
        api.tl_cache_8bit(m, True)
        api.tl_prefill(m, text[:n])
    api.tl_extend(a, text[n:])
    for t in text[n:]:
        api.tl_decode_step(b, t)
    # (a step that completes a block sees its codes, and so may differ: of the last block before the loud token none does)
    first = max(n, loud // 64 * 64)
    for x, y in zip(kv(api, a, shape, 1, first, loud - first), kv(api, b, shape, 1, first, loud - first)):
        # bf16 roundings of differently ordered sums, half a code of either, and half a code of the blocks that steps see as codes and the call does not
        assert far(x, y) <= BF16_TOL + 3 * CODE, far(x, y)
    api.tl_lora_free(a), api.tl_lora_free(b)
    api.tl_model_destroy(model)


def close_to_prefill(api, a, b, shape, n, T, got, want):
    """cached tokens that were all bf16 before the call: everything as a prompt of n + T tokens has it, to within the roundings of differently
    ordered sums"""
    assert far(got, want) <= BF16_TOL, far(got, want)
    for l in range(shape.n_layers):
        for x, y in zip(kv(api, a, shape, l, 0, n + T), kv(api, b, shape, l, 0, n + T)):
            y = held(y, shape)
            done = (n + T) // 64 * 64
            # a code may go to its neighbour, where the twin's value was next to the border: the roundings' share of the values
            assert done == 0 or far(x[:done], y[:done]) <= BF16_TOL + CODE, (l, far(x[:done], y[:done]))
            assert done == n + T or far(x[done:], y[done:]) <= BF16_TOL, l


@pytest.mark.parametrize("name", ["small", "small128"])
@pytest.mark.parametrize("n,T", [(1, 1), (1, 8), (40, 16), (63, 1), (63, 17), (10, 54), (10, 118), (33, 200), (63, 700), (1, 1023)])
@pytest.mark.parametrize("loud", [False, True])
def test_as_one_prompt(api, H, name, n, T, loud):
    shape = synth.SHAPES[name]
    model = loud_model(api, H, shape, 6400, n + T)
    a, b = (module(api, model, shape, 6400) for _ in range(2))
    text = text_of(6400, n + T, shape.vocab, [n + T // 2] if loud else [])
    api.tl_cache_8bit(a, True)
    api.tl_prefill(a, text[:n])
    _, got = api.tl_extend(a, text[n:], shape.vocab)
    _, want = api.tl_prefill(b, text, shape.vocab)
    close_to_prefill(api, a, b, shape, n, T, got, want)
    api.tl_lora_free(a), api.tl_lora_free(b)
    api.tl_model_destroy(model)


WIDE = synth.Shape(2, 4096, 64, 64, 704, 1000, 16, 16.0)


def test_as_one_prompt_in_wide_workgroups(api, H):
    n, T = 60, 520
    assert api.tl_k_attention_cache8_plan(n + T, T, WIDE.n_heads, WIDE.n_heads, WIDE.d_head, 1 << 22)[0] == "rows256"
    model = H.Model(WIDE, 6500, max_tokens=n + T, keep_host=False, device_random=True)
    (a, _), (b, _) = (H.new_lora(model, 6500, b_std=0.01) for _ in range(2))
    text = synth.zipf_tokens(6500, n + T, WIDE.vocab)
    api.tl_cache_8bit(a, True)
    api.tl_prefill(a, text[:n])
    _, got = api.tl_extend(a, text[n:], WIDE.vocab)
    _, want = api.tl_prefill(b, text, WIDE.vocab)
    close_to_prefill(api, a, b, WIDE, n, T, got, want)
    api.tl_lora_free(a), api.tl_lora_free(b)
    model.close()
