"""What the calls on a cache on pages and the drawn token refuse (no GPU needed: nothing is launched)."""
import ctypes as C

import pytest

ARG, SHAPE, WINDOW = -1, -2, -4
P = C.c_void_p(1 << 20)


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


def mem(api, **change):
    m = dict(k=4096, v=8192, table=4, n_pages=9, page_size=16, n_kv_heads=2, d_head=64, n_seqs=3, n_table=5)
    m.update(change)
    return C.byref(api.tl_paged_mem(*m.values()))


def append(api, m, **change):
    a = dict(lengths=P, k=P, ldk=128, v=P, ldv=128, first_row=None, n_rows=3, pos=None, weights=None, positions=None, ldw=0)
    a.update(change)
    return api._lib.tl_k_paged_append(m, *a.values(), None)


def attend(api, m, **change):
    a = dict(lengths=P, max_len=80, q=P, ldq=256, n_heads=4, o=P, ldo=256, w_in=None, w_out=None, ldw=0, workspace=None, elems=0)
    a.update(change)
    return api._lib.tl_k_attention_paged(m, *a.values(), None)


def evict(api, m, **change):
    a = dict(lengths=P, budget=20, recent=5, w=P, p=P, ldw=80, w_out=P, p_out=P, lengths_out=P, workspace=P, elems=3 * 2 * 41)
    a.update(change)
    return api._lib.tl_k_paged_evict(m, *a.values(), None)


@pytest.mark.parametrize("change", [
    dict(k=0), dict(v=0), dict(table=0), dict(k=4104), dict(v=8196), dict(n_pages=0), dict(n_pages=-1), dict(n_pages=2 ** 30 + 1), dict(page_size=0), dict(page_size=8),
    dict(page_size=24), dict(page_size=131072), dict(page_size=-16), dict(n_kv_heads=0), dict(n_kv_heads=5000), dict(d_head=96), dict(d_head=0), dict(n_seqs=-1),
    dict(n_seqs=65536), dict(n_seqs=65535, n_kv_heads=512), dict(n_seqs=65535, n_kv_heads=33), dict(n_table=0), dict(n_table=2 ** 27)])
def test_bad_caches(api, change):
    m = mem(api, **change)
    assert append(api, m) == ARG and attend(api, m) == ARG and evict(api, m) == ARG
    assert "tl_k_paged_evict" in api.tl_last_error()


def test_no_cache(api):
    assert append(api, None) == ARG and attend(api, None) == ARG and evict(api, None) == ARG


def test_nothing_to_do_is_no_error(api):
    assert append(api, mem(api), n_rows=0, lengths=None, k=None, v=None) == 0
    m = mem(api, n_seqs=0)
    assert attend(api, m, lengths=None, q=None, o=None) == 0
    assert evict(api, m, lengths=None, w=None, p=None, w_out=None, p_out=None, lengths_out=None, workspace=None, elems=0) == 0


@pytest.mark.parametrize("change", [
    dict(lengths=None), dict(k=None), dict(v=None), dict(ldk=127), dict(ldv=100), dict(n_rows=-1), dict(n_rows=4), dict(n_rows=2 ** 30 + 1, first_row=P), dict(n_rows=2 ** 23 + 1, first_row=P),
    dict(weights=P), dict(positions=P, ldw=0), dict(weights=P, ldw=-3)])
def test_append(api, change):
    assert append(api, mem(api), **change) == ARG


@pytest.mark.parametrize("change,status", [
    (dict(lengths=None), ARG), (dict(q=None), ARG), (dict(o=None), ARG), (dict(max_len=0), ARG), (dict(max_len=-1), ARG), (dict(max_len=81), WINDOW), (dict(ldq=255), ARG),
    (dict(ldo=255), ARG), (dict(n_heads=3), ARG), (dict(n_heads=0), ARG), (dict(n_heads=65538), ARG), (dict(w_in=P), ARG), (dict(w_out=P, ldw=79), ARG),
    (dict(w_out=P, ldw=80), SHAPE), (dict(w_out=P, ldw=80, workspace=P, elems=3 * 4 * 96 + 23), SHAPE), (dict(w_out=P, ldw=80, elems=1 << 20), SHAPE)])
def test_attention(api, change, status):
    assert attend(api, mem(api), **change) == status


def test_more_weights_than_one_launch_adds_up(api):
    m = mem(api, n_seqs=1024, n_table=2 ** 26)
    n = 2 ** 12 * 1024
    assert attend(api, m, max_len=n + 1, w_out=P, ldw=2 ** 30) == ARG
    assert attend(api, m, max_len=n, w_out=P, ldw=2 ** 30) == SHAPE


@pytest.mark.parametrize("change,status", [
    (dict(lengths=None), ARG), (dict(w=None), ARG), (dict(p=None), ARG), (dict(w_out=None), ARG), (dict(p_out=None), ARG), (dict(lengths_out=None), ARG), (dict(budget=0), ARG),
    (dict(budget=-4), ARG), (dict(recent=-1), ARG), (dict(ldw=0), ARG), (dict(workspace=None), SHAPE), (dict(elems=3 * 2 * 41 - 1), SHAPE),
    (dict(budget=70, elems=3 * 2 * 21 - 1), SHAPE), (dict(budget=200, elems=5), SHAPE)])
def test_evict(api, change, status):
    assert evict(api, mem(api), **change) == status


@pytest.mark.parametrize("change", [
    dict(q=None), dict(k=None), dict(lse=None), dict(w_out=None), dict(T=-1), dict(T=2 ** 30 + 1), dict(n_heads=3), dict(n_heads=0), dict(n_kv=0), dict(n_kv=8192, n_heads=8192),
    dict(d=96), dict(first=-1), dict(ldq=255), dict(ldk=127), dict(ldq=2 ** 25), dict(ldo=9), dict(w_in=P, ldi=9), dict(w_in=C.c_void_p(1 << 21), w_out=C.c_void_p(1 << 21), ldi=10, ldo=11)])
def test_attention_weights(api, change):
    a = dict(q=P, ldq=256, k=P, ldk=128, T=10, n_heads=4, n_kv=2, d=64, first=0, lse=P, w_in=None, ldi=10, w_out=P, ldo=10)
    a.update(change)
    if "w_in" in change and "w_out" in change:
        a["w_in"] = a["w_out"]
    assert api._lib.tl_k_attention_weights(*a.values(), None) == ARG


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(params=None), dict(u=None), dict(choice=None), dict(rows=-1), dict(rows=2 ** 22 + 1), dict(vocab=0), dict(vocab=2 ** 22 + 1), dict(ldl=39), dict(ldp=3), dict(ldp=-4)])
def test_sample(api, change):
    a = dict(logits=P, ldl=40, rows=2, vocab=40, params=P, ldp=4, u=P, choice=P, kept=None, prob=None)
    a.update(change)
    assert api._lib.tl_k_sample(*a.values(), None, 0, None) == ARG


@pytest.mark.parametrize("args", [(0, 1, 4, 4, 64), (2 ** 30 + 1, 1, 4, 4, 64), (5, 0, 4, 4, 64), (5, 1, 3, 2, 64), (5, 1, 4, 0, 64), (5, 1, 4, 4, 80), (5, 65536, 4, 4, 64),
                                  (5, 65535, 512, 4, 64), (5, 65535, 68, 4, 64)])
def test_bad_plans(api, args):
    with pytest.raises(api.TlError):
        api.tl_k_attention_paged_plan(*args)


def test_plan_stays_within_the_workspace(api):
    for max_len in (1, 200, 4096, 131072, 2 ** 30):
        for n_seqs in (1, 7, 500):
            for heads, kv in ((4, 4), (32, 8), (40, 1)):
                for elems in (0, 1000, 1 << 16, 1 << 24):
                    n, used = api.tl_k_attention_paged_plan(max_len, n_seqs, heads, kv, 128, False, elems)
                    assert 1 <= n <= 128 and used <= elems
                    n, used = api.tl_k_attention_paged_plan(max_len, n_seqs, heads, kv, 128, True, elems)
                    least = n_seqs * heads * ((max_len + 31) // 32 * 32)
                    assert 1 <= n <= 128 and used >= least and (used <= elems or n == 1)


def test_set_sampling_without_a_module(api):
    assert api._lib.tl_set_sampling(None, None) == ARG
