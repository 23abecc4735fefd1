"""Device memory of the caches: a call that fails for want of it gives back what it had taken, and the 8-bit cache takes the place of the
buffers of tl_cache_reuse."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2401_11504_amd import synth  # noqa: E402
from test_gpu_kernels import H, api  # noqa: E402,F401

MB = 1 << 20
SHAPE = synth.Shape(8, 256, 4, 64, 64, 64, 8, 8.0)
N = 1 << 20            # tokens: 512 MB of codes and 1.5 GB of bf16 rows a layer


def free():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0]


@pytest.fixture(scope="module")
def model(H):
    m = H.Model(SHAPE, 6700, max_tokens=N, keep_host=False)
    yield m
    m.close()


def fill_up_to(left):
    """tensors that leave about `left` bytes of the device's memory"""
    held = []
    while free() > left + 64 * MB:
        n = min(free() - left - 32 * MB, 16 << 30)
        held.append(torch.empty(n, dtype=torch.uint8, device="cuda"))
    return held


def oom(api, f, *args):
    with pytest.raises(api.TlError) as e:
        f(*args)
    assert e.value.status == -8, e.value


def test_out_of_memory(api, H, model):
    """1.3 and 3 GB are enough for some of the buffers and not for all (8 layers of 512 MB and 1 GB beside them; 8 of 1.5 GB)"""
    a, b, c = (H.new_lora(model, 6700, b_std=0.01)[0] for _ in range(3))
    text = synth.zipf_tokens(6700, 200, SHAPE.vocab)
    api.tl_cache_8bit(c, True)
    api.tl_cache_reuse(c, True)
    calls = ((a, api.tl_cache_8bit, True), (b, api.tl_cache_reuse, True), (c, api.tl_cache_8bit, False))    # the last: bf16 buffers again
    for m, _, _ in calls:
        api.tl_prefill(m, text[:100])
    held = fill_up_to(3000 * MB)
    for left in (3000, 1300):
        if left == 1300:
            held.append(torch.empty(1700 * MB, dtype=torch.uint8, device="cuda"))
        for m, f, on in calls:
            before = free()
            for _ in range(3):
                oom(api, f, m, on)
                assert free() >= before - 2 * MB
            assert api.tl_kv_length(m) == 100                    # as it was
    for m, _, _ in calls:
        api.tl_decode_step(m, text[100])
    del held
    torch.cuda.empty_cache()
    for m, f, on in calls:
        f(m, on)
        api.tl_prefill(m, text[:100])
        nxt, logits = api.tl_decode_step(m, text[100], SHAPE.vocab)
        assert np.isfinite(logits).all()
        api.tl_lora_free(m)


def test_buffers_of_reuse_are_given_back(api, H, model):
    a, _ = H.new_lora(model, 6700, b_std=0.01)
    b, _ = H.new_lora(model, 6700, b_std=0.01)
    text = synth.zipf_tokens(6700, 200, SHAPE.vocab)
    api.tl_cache_8bit(b, True)
    start = free()
    api.tl_cache_reuse(a, True)
    assert start - free() >= (8 * 1536 - 64) * MB                 # (less what the allocator had kept of earlier frees)
    for m in (a, b):
        api.tl_prefill(m, text[:100])
    api.tl_cache_8bit(a, True)                                   # the cache moves along
    assert start - free() <= 8 * 512 * MB + 1200 * MB
    for i in range(100, 104):
        xa, xb = api.tl_decode_step(a, text[i], SHAPE.vocab), api.tl_decode_step(b, text[i], SHAPE.vocab)
        assert xa[0] == xb[0] and np.array_equal(xa[1], xb[1])
    api.tl_chunk_update(a, text[:32], 0, 1e-3)
    assert api.tl_kv_length(a) == 104                            # reuse is still on
    api.tl_cache_8bit(a, False)
    api.tl_prefill(a, text[:100])
    api.tl_chunk_update(a, text[:32], 0, 1e-3)
    assert api.tl_kv_length(a) == 100
    api.tl_decode_step(a, text[100])
    api.tl_lora_free(a), api.tl_lora_free(b)
