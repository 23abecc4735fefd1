"""The ranges that the attention over pages plans (host only): no more than a wave joins, as many where one head has many keys, and what the workspace is needed for."""
import pytest

MOST = 64


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


@pytest.mark.parametrize("weights", [False, True])
def test_no_more_ranges_than_a_wave_joins(api, weights):
    seen = set()
    for max_len in (1, 127, 128, 129, 512, 513, 2048, 2049, 4096, 10000, 50001, 131072, 2 ** 20, 2 ** 30):
        for n_seqs in (1, 2, 7, 33, 64, 500, 65535):
            for heads, kv in ((1, 1), (4, 4), (32, 8), (40, 1), (32, 32)):
                for elems in (0, 1000, 1 << 16, 1 << 24, 1 << 40):
                    for d in (64, 128):
                        n, used = api.tl_k_attention_paged_plan(max_len, n_seqs, heads, kv, d, weights, elems)
                        assert 1 <= n <= MOST and n <= -(-max_len // 128)
                        rows = n_seqs * heads
                        scores = rows * ((max_len + 31) // 32 * 32) if weights else 0
                        joined = (rows * n * 2 + 3) // 4 * 4 if weights or n > 1 else 0
                        assert used == scores + joined + (rows * n * d if n > 1 else 0)
                        assert used <= elems or (weights and n == 1)
                        seen.add(n)
    assert {1, 2, 8, MOST} <= seen


def test_all_of_them_for_one_head(api):
    assert api.tl_k_attention_paged_plan(131072, 1, 1, 1, 128, False, 1 << 24)[0] == MOST
    assert api.tl_k_attention_paged_plan(131072, 1, 1, 1, 64, True, 1 << 24)[0] == MOST
