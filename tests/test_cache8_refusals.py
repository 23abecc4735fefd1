"""What the calls on the 8-bit cache and the choice of a token refuse (no GPU needed: nothing is launched)."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, WINDOW = -1, -4


@pytest.fixture(scope="module")
def api():
    from paper_2401_11504_amd import api
    return api


def mem(api, **change):
    m = dict(k=4096, v=8192, k_scale=4, v_scale=8, k_tail=16, v_tail=32, n_kv_heads=2, d_head=64, capacity=100)
    m.update(change)
    return api.tl_cache8_mem(*m.values())


P = C.c_void_p(1 << 20)
BAD_MEM = [dict(k=0), dict(v=0), dict(k_scale=0), dict(v_scale=0), dict(k_tail=0), dict(v_tail=0), dict(k=8), dict(v=24), dict(k_tail=2), dict(v_tail=4),
           dict(n_kv_heads=0), dict(n_kv_heads=-1), dict(n_kv_heads=5000), dict(d_head=96), dict(d_head=0), dict(capacity=0), dict(capacity=2 ** 30 + 1), dict(capacity=-5)]


@pytest.mark.parametrize("change", BAD_MEM)
def test_bad_caches(api, change):
    m = C.byref(mem(api, **change))
    assert api._lib.tl_k_cache8_append(m, 0, P, 128, P, 128, 1, None) == ARG
    assert api._lib.tl_k_cache8_read(m, 1, 0, 1, P, 128, P, 128, None) == ARG
    assert api._lib.tl_k_attention_cache8(m, 1, P, 128, 1, 2, P, 128, None, 0, None) == ARG
    assert "tl_k_attention_cache8" in api.tl_last_error()


def test_no_cache(api):
    assert api._lib.tl_k_cache8_append(None, 0, P, 128, P, 128, 1, None) == ARG
    assert api._lib.tl_k_cache8_read(None, 1, 0, 1, P, 128, P, 128, None) == ARG
    assert api._lib.tl_k_attention_cache8(None, 1, P, 128, 1, 2, P, 128, None, 0, None) == ARG


@pytest.mark.parametrize("n_cached,k,ldk,v,ldv,n_new,status", [
    (0, None, 128, P, 128, 1, ARG), (0, P, 128, None, 128, 1, ARG), (-1, P, 128, P, 128, 1, ARG), (0, P, 128, P, 128, -1, ARG),
    (0, P, 127, P, 128, 2, ARG), (0, P, 128, P, 127, 2, ARG), (100, P, 128, P, 128, 1, WINDOW), (0, P, 128, P, 128, 101, WINDOW),
    (2 ** 31 - 1, P, 128, P, 128, 2 ** 31 - 1, WINDOW)])
def test_append(api, n_cached, k, ldk, v, ldv, n_new, status):
    assert api._lib.tl_k_cache8_append(C.byref(mem(api)), n_cached, k, ldk, v, ldv, n_new, None) == status


@pytest.mark.parametrize("n_cached,first,n,k,ldk,status", [
    (10, 0, 11, P, 128, WINDOW), (101, 0, 1, P, 128, WINDOW), (10, -1, 1, P, 128, ARG), (10, 0, -1, P, 128, ARG), (10, 0, 2, P, 100, ARG),
    (10, 0, 1, None, 128, ARG), (10, 2 ** 31 - 1, 2 ** 31 - 1, P, 128, WINDOW)])
def test_read(api, n_cached, first, n, k, ldk, status):
    assert api._lib.tl_k_cache8_read(C.byref(mem(api)), n_cached, first, n, k, ldk, P, 128, None) == status


@pytest.mark.parametrize("n_keys,q,ldq,rows,heads,o,ldo,status", [
    (1, None, 128, 1, 2, P, 128, ARG), (1, P, 128, 1, 2, None, 128, ARG), (0, P, 128, 0, 2, P, 128, ARG), (5, P, 128, -1, 2, P, 128, ARG),
    (5, P, 128, 1, 3, P, 128, ARG), (5, P, 128, 1, 0, P, 128, ARG), (5, P, 255, 2, 4, P, 256, ARG), (5, P, 256, 2, 4, P, 255, ARG),
    (101, P, 128, 1, 2, P, 128, WINDOW), (5, P, 128, 6, 2, P, 128, WINDOW), (5, P, 128, 1, 65538, P, 128, ARG)])
def test_attention(api, n_keys, q, ldq, rows, heads, o, ldo, status):
    assert api._lib.tl_k_attention_cache8(C.byref(mem(api)), n_keys, q, ldq, rows, heads, o, ldo, None, 0, None) == status


@pytest.mark.parametrize("args", [(0, 1, 2, 2, 64), (2 ** 30 + 1, 1, 2, 2, 64), (5, 6, 2, 2, 64), (5, 0, 2, 2, 64), (5, 1, 3, 2, 64), (5, 1, 2, 0, 64), (5, 1, 2, 2, 80)])
def test_plan(api, args):
    with pytest.raises(api.TlError):
        api.tl_k_attention_cache8_plan(*args)


def test_plan_stays_within_the_workspace(api):
    for n_keys in (1, 200, 4096, 131072):
        for rows in (1, 5, 40, 400):
            if rows > n_keys:
                continue
            for heads, kv in ((4, 4), (32, 8), (20, 1)):
                for elems in (0, 1000, 1 << 16, 1 << 24):
                    name, n, used = api.tl_k_attention_cache8_plan(n_keys, rows, heads, kv, 128, elems)
                    assert 1 <= n <= 64 and used <= elems and name


@pytest.mark.parametrize("tokens,ldt,rows,n,vocab,add,counts,ldc", [
    (None, 4, 1, 4, 10, 0, P, 10), (P, 4, 1, 4, 10, 0, None, 10), (P, 4, -1, 4, 10, 0, P, 10), (P, 4, 1, -4, 10, 0, P, 10), (P, 4, 1, 4, 0, 0, P, 10),
    (P, 4, 1, 4, 10, 2, P, 10), (P, 4, 1, 4, 10, -2, P, 10), (P, 3, 2, 4, 10, 0, P, 10), (P, 4, 2, 4, 10, 0, P, 9),
    (P, 4, 1, 2 ** 30 + 1, 10, 0, P, 10), (P, 4, 1, 4, 2 ** 30 + 1, 0, P, 10)])
def test_counts(api, tokens, ldt, rows, n, vocab, add, counts, ldc):
    assert api._lib.tl_k_token_counts(tokens, ldt, rows, n, vocab, add, counts, ldc, None) == ARG


GOOD = dict(logits=P, ldl=40, rows=2, vocab=40, counts=P, ldc=40, repetition=1.0, presence=0.0, frequency=0.0, bias=P, ldb=40, allowed=P, lda=2, out=P,
            ldo=40, choice=P)


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(ldl=39), dict(rows=-1), dict(vocab=0), dict(vocab=2 ** 30 + 1, rows=1), dict(ldc=39), dict(ldb=39), dict(lda=1), dict(ldo=39), dict(ldo=0), dict(ldl=41),
    dict(repetition=0.0), dict(repetition=-1.0), dict(repetition=float("nan")), dict(repetition=float("inf")), dict(presence=float("nan")),
    dict(frequency=float("inf"))])
def test_choose(api, change):
    a = dict(GOOD, **change)
    assert api._lib.tl_k_choose(*a.values(), None, 0, None) == ARG
