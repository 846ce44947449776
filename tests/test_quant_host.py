"""Refusals of the products in 8-bit integers: every argument is looked at on the host before anything is launched (no GPU needed: none of the
addresses below is ever read)."""
import ctypes as C

import pytest

from paper_2511_11641_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    return B.load()


@pytest.fixture()
def ctx(lib):
    h = C.c_void_p()
    assert lib.ecospa_create(C.byref(h), None) == B.OK
    yield h
    lib.ecospa_destroy(h)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), B.ERR_NULL), (dict(q=None), B.ERR_NULL), (dict(scale=None), B.ERR_NULL), (dict(dtype=2), B.ERR_DTYPE), (dict(dtype=-1), B.ERR_DTYPE),
    (dict(rows=0), B.ERR_SHAPE), (dict(rows=(1 << 30) + 1), B.ERR_SHAPE), (dict(cols=0), B.ERR_SHAPE), (dict(cols=12), B.ERR_SHAPE), (dict(ld=56), B.ERR_SHAPE), (dict(ld_q=48), B.ERR_SHAPE),
    (dict(ld=68), B.ERR_ALIGN), (dict(ld_q=72), B.ERR_ALIGN), (dict(x=264), B.ERR_ALIGN), (dict(q=520), B.ERR_ALIGN),
], ids=str)
def test_rows_are_refused(lib, ctx, change, code):
    a = dict(rows=3, cols=64, dtype=B.BF16, x=256, ld=64, q=512, ld_q=64, scale=1024) | change
    assert lib.ecospa_quant_rows(ctx, *a.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(A=None), B.ERR_NULL), (dict(sa=None), B.ERR_NULL), (dict(Bm=None), B.ERR_NULL), (dict(sb=None), B.ERR_NULL), (dict(C=None), B.ERR_NULL),
    (dict(act=3), B.ERR_DTYPE), (dict(act=-2), B.ERR_DTYPE), (dict(M=0), B.ERR_SHAPE), (dict(N=0), B.ERR_SHAPE), (dict(K=0), B.ERR_SHAPE),
    (dict(K=131072, lda=131072, ldb=131072), B.ERR_SHAPE), (dict(lda=48), B.ERR_SHAPE), (dict(ldb=48), B.ERR_SHAPE), (dict(ldc=24), B.ERR_SHAPE),
    (dict(lda=1 << 24), B.ERR_SHAPE), (dict(ldb=1 << 24), B.ERR_SHAPE), (dict(ldc=1 << 23), B.ERR_SHAPE),
    (dict(K=40), B.ERR_ALIGN), (dict(N=28), B.ERR_ALIGN), (dict(N=24, act=B.ACT_SWIGLU), B.ERR_ALIGN), (dict(lda=72), B.ERR_ALIGN), (dict(ldb=72), B.ERR_ALIGN),
    (dict(ldc=36), B.ERR_ALIGN), (dict(A=264), B.ERR_ALIGN), (dict(Bm=264), B.ERR_ALIGN), (dict(C=264), B.ERR_ALIGN), (dict(sb=260), B.ERR_ALIGN),
    (dict(bias=258), B.ERR_ALIGN), (dict(sa=258), B.ERR_ALIGN),
], ids=str)
def test_products_are_refused(lib, ctx, change, code):
    a = dict(M=5, N=32, K=64, A=256, lda=64, sa=512, Bm=1024, ldb=64, sb=2048, bias=None, act=B.ACT_NONE, C=4096, ldc=32) | change
    assert lib.ecospa_contract_quant(ctx, *a.values()) == code


def test_without_a_context(lib):
    assert lib.ecospa_quant_rows(None, 3, 64, B.BF16, 256, 64, 512, 64, 1024) == B.ERR_NULL
    assert lib.ecospa_contract_quant(None, 5, 32, 64, 256, 64, 512, 1024, 64, 2048, None, B.ACT_NONE, 4096, 32) == B.ERR_NULL
