"""Device memory of the caches: a call that fails for want of it gives back what it had taken."""
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
