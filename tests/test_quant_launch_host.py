"""Calls whose work does not fit a launch (2^32 work-items and more) are refused on the host before anything is launched (no GPU needed: none of the addresses
below is ever read)."""
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


def cache(Bsz, h, h_kv, cap, width=16, block=16):
    return B.QuantCacheDesc(Bsz, h, h_kv, width, width, cap, cap, block, 0.125, 4096, 8192, h_kv * cap * width, cap * width, width, h_kv * cap * width, cap * width, width,
                            16384, 32768, 65536)


@pytest.mark.parametrize("Bsz,h,h_kv,L,q", [(65535, 1, 1, 8192, None), (65535, 1, 1, 8190, 512), (4096, 16, 1, 16384, 512)], ids=["blocks", "blocks and queries", "queries"])
def test_appends(lib, ctx, Bsz, h, h_kv, L, q):
    c = cache(Bsz, h, h_kv, 1 << 20, width=16 if h == 1 else 64)
    width = c.kp_qk * (h + 2 * h_kv)
    assert lib.ecospa_quant_cache_append(ctx, C.byref(c), L, 256, width, None, None, None, 0, q, h * c.kp_qk) == B.ERR_SHAPE


@pytest.mark.parametrize("Bsz,h,h_kv,L,width", [(65535, 1, 1, 16384, 16), (32760, 2, 1, 16384, 128), (1, 1, 1, 1 << 27, 16)])
def test_attention(lib, ctx, Bsz, h, h_kv, L, width):
    c = cache(Bsz, h, h_kv, 1 << 10, width=width)
    n = h * width
    assert lib.ecospa_quant_cache_attn(ctx, C.byref(c), L, 256, n, None, 0, None, 512, n, None) == B.ERR_SHAPE


@pytest.mark.parametrize("M,N,K,act", [((1 << 31) - 1, 8, 16, B.ACT_NONE), (1 << 30, 2048, 64, B.ACT_NONE), (1 << 30, 2048, 2048, B.ACT_SWIGLU),
                                       (1 << 21, 1 << 20, 4096, B.ACT_GELU_TANH), (1 << 30, 1 << 20, 2048, B.ACT_NONE)])
def test_products(lib, ctx, M, N, K, act):
    assert lib.ecospa_contract_quant(ctx, M, N, K, 256, K, 512, 1024, K, 2048, None, act, 4096, N) == B.ERR_SHAPE
