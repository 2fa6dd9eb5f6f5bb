"""What the group norms and the products of few rows refuse, through the C ABI and without a GPU: these checks stand in front of the first
CUDA call, so the pointers are never followed."""
import ctypes as C

import pytest

from paper_2501_04304_b200 import binding as b
from test_encoder_refusals import ALIGNMENT, INVALID, PTR, UNSUPPORTED, rows

WORKSPACE = 4
BIG = 1 << 24


def norm(X=None, add=None, ld_add=64, gamma=None, beta=None, Y=None, dtype=0, B=2, P=1 << 20, c=64, groups=8, eps=1e-5, act=0, ws=PTR, size=BIG):
    X, Y = X or rows(), Y or rows()
    return b.lib().dgq_group_norm(C.byref(X), C.c_void_p(add), C.c_int64(ld_add), C.c_void_p(gamma), C.c_void_p(beta), C.byref(Y), dtype, B, P, c, groups,
                                  C.c_float(eps), act, C.c_void_p(ws), C.c_size_t(size), None)


@pytest.mark.parametrize("change,status", [
    (dict(X=rows(ptr=None)), INVALID), (dict(Y=rows(ptr=None)), INVALID), (dict(B=0), INVALID), (dict(P=0), INVALID), (dict(P=-1), INVALID), (dict(c=0), INVALID),
    (dict(groups=0), INVALID), (dict(groups=7), INVALID), (dict(dtype=2), INVALID), (dict(act=2), INVALID), (dict(act=-1), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=-1e-5), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(add=PTR, ld_add=-64), INVALID),
    (dict(X=rows(token=0)), INVALID), (dict(Y=rows(token=0)), INVALID), (dict(Y=rows(batch=0)), INVALID), (dict(Y=rows(token=56)), INVALID),
    (dict(X=rows(token=-64)), INVALID), (dict(X=rows(ptr=PTR + 8)), ALIGNMENT), (dict(Y=rows(ptr=PTR + 2)), ALIGNMENT), (dict(X=rows(token=68)), ALIGNMENT),
    (dict(Y=rows(batch=4100)), ALIGNMENT), (dict(ws=PTR + 16), ALIGNMENT), (dict(c=60, groups=6), UNSUPPORTED), (dict(c=4104), UNSUPPORTED), (dict(B=65536), UNSUPPORTED),
    (dict(P=(1 << 30) + 1), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(size=64), WORKSPACE),
], ids=str)
def test_group_norm(change, status):
    assert norm(**change) == status


def test_workspace_bytes():
    def need(B, P, c, groups, quantize=1):
        n = C.c_size_t(7)
        return b.lib().dgq_group_norm_workspace_bytes(B, P, c, groups, quantize, C.byref(n)), n.value

    assert need(2, 4096, 320, 32)[0] == 0 and 0 < need(2, 4096, 320, 32)[1] <= 1 << 20
    assert need(2, 64, 1280, 32, 0) == (0, 0) and need(1, 1 << 18, 128, 32, 0)[1] > 0
    for bad in ((0, 1, 8, 1), (1, 0, 8, 1), (1, 1, 0, 1), (1, 1, 8, 0), (1, 1, 8, 3)):
        assert need(*bad)[0] == INVALID
    for bad in ((1, 1, 12, 1), (1, 1, 4104, 1), (65536, 1, 8, 1), (2 ** 31 - 1, 1, 8, 1), (1, (1 << 30) + 1, 8, 1), (1, 2 ** 31 - 1, 8, 1)):
        assert need(*bad)[0] == UNSUPPORTED
    assert b.lib().dgq_group_norm_workspace_bytes(1, 1, 8, 1, 1, None) == INVALID
    for B in (1, 7, 300, 65535):
        assert need(B, 1000, 64, 8)[1] >= B * 8 * 16


def test_codes():
    x = rows()
    assert b.lib().dgq_group_norm_quantize(None, 0, 0, C.byref(x), None, C.c_int64(0), None, None, 0, 1, 1, 1, C.c_float(1e-5), 0, C.c_void_p(PTR), C.c_void_p(PTR),
                                           C.c_size_t(BIG), None) == INVALID


def test_few():
    lib = b.lib()
    out = C.c_void_p(None)

    def prepare(W=PTR, N=16, K=64, group=64, to=out):
        return lib.dgq_few_weight_prepare(C.c_void_p(W), N, K, group, C.byref(to) if to is not None else None, None)

    for bad in (dict(W=None), dict(N=0), dict(K=0), dict(K=-8), dict(group=16), dict(group=0), dict(group=96), dict(to=None)):
        assert prepare(**bad) == INVALID, bad
    for bad in (dict(K=60), dict(N=1 << 20), dict(K=1 << 20)):
        assert prepare(**bad) == UNSUPPORTED, bad
    assert lib.dgq_few_weight_from_codes(None, C.c_void_p(PTR), 16, 64, 64, C.byref(out), None) == INVALID
    assert lib.dgq_few_weight_from_codes(C.c_void_p(PTR), None, 16, 64, 64, C.byref(out), None) == INVALID
    assert lib.dgq_few_weight_export(None, None, None) == INVALID
    assert lib.dgq_few_weight_destroy(None) == 0
    assert lib.dgq_linear_few(None, C.c_void_p(PTR), C.c_int64(64), 0, 1, 0, None, C.c_void_p(PTR), C.c_int64(16), None) == INVALID
    assert out.value is None


def test_large_integers():
    with pytest.raises(ValueError, match="32 bits"):
        b.native().linear_few(0, 2 ** 31, 64, None, 0, None, None, None)
    with pytest.raises(ValueError, match="32 bits"):
        b.native().group_norm(None, 2 ** 32 + 8, None, None, 1e-5, 0, None, None, None, None)


@pytest.mark.parametrize("B,P,batch,token", [(2, 1 << 20, 4096, 256), (2, 16, 64, 64), (2, 16, 960, 64), (3, 16, 512, 256), (2, 1, 56, 64), (2, 3, 8, 64), (4, 3, 64, 192),
                                             (65535, 2, 64, 65534 * 64), (3, 1 << 30, 1 << 36, 72), (2, 4, 176, 128)])
def test_images_that_overlap(B, P, batch, token):
    assert norm(Y=rows(batch=batch, token=token), B=B, P=P) == INVALID
