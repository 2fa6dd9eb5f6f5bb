"""What the calls for attention over encoder states and over the 8-bit cache refuse, through the C ABI and without a GPU: every check
stands in front of the first CUDA call, so the pointers are never followed."""
import ctypes as C

import pytest

from paper_2501_04304_b200 import binding as b


class Rows(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n_pages", C.c_int),
                ("n_heads", C.c_int), ("page", C.c_int), ("d", C.c_int)]


PTR = 0x10000
INVALID, ALIGNMENT, UNSUPPORTED = 1, 2, 3


def rows(ptr=PTR, batch=4096, token=256, head=64):
    return Rows(ptr, batch, token, head)


def encoder(Q=None, K=None, V=None, O=None, dtype=0, B=2, Hq=4, Hkv=2, nq=3, nk=5, d=64, scale=0.1):
    r = [x if x is not None else rows() for x in (Q, K, V, O)]
    return b.lib().dgq_encoder_attn(*[C.byref(x) for x in r], C.c_int(dtype), C.c_int(B), C.c_int(Hq), C.c_int(Hkv), C.c_int(nq), C.c_int(nk),
                                    C.c_int(d), C.c_float(scale), None, None)


def cache(**change):
    c = Cache(PTR, PTR, PTR, PTR, 10, 2, 16, 64)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def cached(c=None, Q=None, O=None, dtype=0, B=2, Hq=4, n_rows=6, q_start=None, max_nq=3, table=PTR, max_pages=4, lens=PTR, scale=0.1):
    c, Q, O = c or cache(), Q or rows(), O or rows()
    return b.lib().dgq_cached_attn(C.byref(c), C.byref(Q), C.byref(O), C.c_int(dtype), C.c_int(B), C.c_int(Hq), C.c_int64(n_rows), C.c_void_p(q_start),
                                   C.c_int(max_nq), C.c_void_p(table), C.c_int(max_pages), C.c_void_p(lens), C.c_int(0), C.c_float(scale), None)


def write(c=None, K=None, V=None, dtype=0, T=5, slots=PTR, name="dgq_kv_write"):
    c, K, V = c or cache(), K or rows(), V or rows()
    if name == "dgq_kv_read":
        return b.lib().dgq_kv_read(C.byref(c), C.c_void_p(slots), C.c_int64(T), C.byref(K), C.byref(V), C.c_int(dtype), None)
    return b.lib().dgq_kv_write(C.byref(c), C.byref(K), C.byref(V), C.c_int(dtype), C.c_int64(T), C.c_void_p(slots), None)


@pytest.mark.parametrize("change,status", [
    (dict(Q=rows(ptr=None)), INVALID), (dict(O=rows(ptr=None)), INVALID), (dict(B=0), INVALID), (dict(nq=0), INVALID), (dict(nk=-1), INVALID),
    (dict(Hq=3), INVALID), (dict(dtype=2), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(K=rows(token=0)), INVALID), (dict(O=rows(batch=0)), INVALID), (dict(O=rows(head=0)), INVALID), (dict(V=rows(head=-64)), INVALID),
    (dict(K=rows(ptr=PTR + 8)), ALIGNMENT), (dict(V=rows(token=260)), ALIGNMENT), (dict(d=60), UNSUPPORTED), (dict(d=168), UNSUPPORTED),
    (dict(K=rows(batch=1 << 38)), UNSUPPORTED),
], ids=str)
def test_encoder_attention(change, status):
    assert encoder(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(c=cache(k=None)), INVALID), (dict(c=cache(n_pages=0)), INVALID), (dict(c=cache(page=24)), UNSUPPORTED), (dict(c=cache(page=256)), UNSUPPORTED),
    (dict(c=cache(d=4)), UNSUPPORTED), (dict(c=cache(d=176)), UNSUPPORTED), (dict(c=cache(n_pages=1 << 27)), UNSUPPORTED), (dict(c=cache(v=PTR + 4)), ALIGNMENT),
    (dict(Hq=3), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(max_nq=0), INVALID), (dict(max_pages=0), INVALID),
    (dict(q_start=PTR, n_rows=0), INVALID), (dict(Q=rows(token=12)), ALIGNMENT), (dict(O=rows(token=0)), INVALID), (dict(dtype=-1), INVALID),
    (dict(max_pages=1 << 28), UNSUPPORTED), (dict(scale=float("-inf")), INVALID),
], ids=str)
def test_cached_attention(change, status):
    assert cached(**change) == status


@pytest.mark.parametrize("name", ["dgq_kv_write", "dgq_kv_read"])
@pytest.mark.parametrize("change,status", [
    (dict(c=cache(v_scale=None)), INVALID), (dict(T=0), INVALID), (dict(slots=None), INVALID), (dict(K=rows(ptr=None)), INVALID), (dict(dtype=5), INVALID),
    (dict(V=rows(head=4)), ALIGNMENT), (dict(K=rows(token=0)), INVALID), (dict(c=cache(page=8)), UNSUPPORTED),
], ids=str)
def test_rows_in_and_out(name, change, status):
    assert write(name=name, **change) == status


def test_values_out_do_not_broadcast():
    assert write(K=rows(head=0), name="dgq_kv_read") == INVALID


def test_null_structs():
    lib = b.lib()
    assert lib.dgq_encoder_attn(None, None, None, None, 0, 1, 1, 1, 1, 1, 8, C.c_float(1), None, None) == INVALID
    assert lib.dgq_kv_write(None, None, None, 0, C.c_int64(1), None, None) == INVALID


def test_plan():
    def plan(lens=PTR, new=PTR + 64, B=4, free=PTR + 128, n_free=3, table=PTR + 256, max_pages=2, page=16, start=PTR + 512, kv=PTR + 1024, slots=PTR + 2048,
             n_slots=8, used=PTR + 4096):
        return b.lib().dgq_kv_plan(*[C.c_void_p(x) for x in (lens, new)], B, C.c_void_p(free), n_free, C.c_void_p(table), max_pages, page, C.c_void_p(start),
                                   C.c_void_p(kv), C.c_void_p(slots), n_slots, C.c_void_p(used), None)

    assert plan(page=48) == UNSUPPORTED
    for bad in (dict(lens=None), dict(B=0), dict(free=None), dict(table=None), dict(max_pages=0), dict(slots=None), dict(n_slots=-1), dict(used=None),
                dict(kv=PTR), dict(kv=PTR + 12), dict(start=PTR + 64 - 4), dict(start=PTR)):
        assert plan(**bad) == INVALID, bad
