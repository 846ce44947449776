"""Refusals of the caches of 8-bit floats and of drawing tokens: every argument is looked at on the host before anything is launched (no GPU
needed: none of the addresses below is ever read)."""
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


def cache(**kw):
    c = B.QuantCacheDesc(2, 8, 4, 32, 48, 100, 90, 32, 0.125, 4096, 8192, 4 * 100 * 32, 100 * 32, 32, 4 * 100 * 48, 100 * 48, 48, 16384, 32768, 65536)
    for n, x in kw.items():
        setattr(c, n, x)
    return c


BAD_CACHES = [
    (dict(k=None), B.ERR_NULL), (dict(v=None), B.ERR_NULL), (dict(lens=None), B.ERR_NULL), (dict(k_scale=None), B.ERR_NULL), (dict(v_scale=None), B.ERR_NULL),
    (dict(B=0), B.ERR_SHAPE), (dict(h=0), B.ERR_SHAPE), (dict(h=6), B.ERR_SHAPE), (dict(h_kv=0), B.ERR_SHAPE), (dict(h=2), B.ERR_SHAPE),
    (dict(cap=0, own_max=0), B.ERR_SHAPE), (dict(own_max=101), B.ERR_SHAPE), (dict(own_max=-1), B.ERR_SHAPE),
    (dict(kp_qk=24), B.ERR_SHAPE), (dict(kp_qk=0), B.ERR_SHAPE), (dict(kp_vo=144, v_st=144), B.ERR_SHAPE), (dict(kp_vo=8), B.ERR_SHAPE),
    (dict(block=8), B.ERR_SHAPE), (dict(block=48), B.ERR_SHAPE), (dict(block=256), B.ERR_SHAPE), (dict(block=0), B.ERR_SHAPE),
    (dict(scale=0.0), B.ERR_SHAPE), (dict(scale=-1.0), B.ERR_SHAPE), (dict(scale=float("nan")), B.ERR_SHAPE), (dict(scale=float("inf")), B.ERR_SHAPE),
    (dict(k_st=16), B.ERR_SHAPE), (dict(v_st=32), B.ERR_SHAPE), (dict(k_st=1 << 25), B.ERR_SHAPE), (dict(k_sb=-16), B.ERR_SHAPE), (dict(v_sh=-16), B.ERR_SHAPE),
    (dict(k=4104), B.ERR_ALIGN), (dict(v=8200), B.ERR_ALIGN), (dict(k_st=40), B.ERR_ALIGN), (dict(v_sb=8), B.ERR_ALIGN), (dict(k_scale=16386), B.ERR_ALIGN),
    (dict(lens=65537), B.ERR_ALIGN), (dict(B=40000), B.ERR_SHAPE),
]


@pytest.mark.parametrize("change,code", BAD_CACHES, ids=[str(c) for c, _ in BAD_CACHES])
def test_caches_are_refused(lib, ctx, change, code):
    c = cache(**change)
    assert lib.ecospa_quant_cache_attn(ctx, C.byref(c), 1, 256, 256, None, 0, None, 512, 384, None) == code
    assert lib.ecospa_quant_cache_attn_workspace_bytes(C.byref(c), 1) == 0
    assert lib.ecospa_quant_cache_append(ctx, C.byref(c), 1, 256, 576, None, None, None, 0, 512, 256) == code


def test_without_a_cache_or_a_context(lib, ctx):
    c = cache()
    assert lib.ecospa_quant_cache_attn(ctx, None, 1, 256, 256, None, 0, None, 512, 384, None) == B.ERR_NULL
    assert lib.ecospa_quant_cache_append(ctx, None, 1, 256, 576, None, None, None, 0, 512, 256) == B.ERR_NULL
    assert lib.ecospa_quant_cache_attn_workspace_bytes(None, 1) == 0
    assert lib.ecospa_quant_cache_attn(None, C.byref(c), 1, 256, 256, None, 0, None, 512, 384, None) == B.ERR_NULL
    assert lib.ecospa_quant_cache_append(None, C.byref(c), 1, 256, 576, None, None, None, 0, 512, 256) == B.ERR_NULL


@pytest.mark.parametrize("change,code", [
    (dict(q=None), B.ERR_NULL), (dict(o=None), B.ERR_NULL), (dict(o_in=2048), B.ERR_NULL), (dict(lse_in=2048), B.ERR_NULL),
    (dict(L=0), B.ERR_SHAPE), (dict(L=1 << 27), B.ERR_SHAPE), (dict(ld_q=248), B.ERR_SHAPE), (dict(ld_o=376), B.ERR_SHAPE), (dict(o_in=2048, lse_in=4096, ld_oi=376), B.ERR_SHAPE),
    (dict(q=264), B.ERR_ALIGN), (dict(o=520), B.ERR_ALIGN), (dict(ld_q=260), B.ERR_ALIGN), (dict(ld_o=388), B.ERR_ALIGN), (dict(lse=1026), B.ERR_ALIGN),
    (dict(o_in=2056, lse_in=4096, ld_oi=384), B.ERR_ALIGN), (dict(o_in=2048, lse_in=4098, ld_oi=384), B.ERR_ALIGN), (dict(o_in=2048, lse_in=4096, ld_oi=388), B.ERR_ALIGN),
], ids=str)
def test_attention_refusals(lib, ctx, change, code):
    a = dict(L=2, q=256, ld_q=256, o_in=None, ld_oi=0, lse_in=None, o=512, ld_o=384, lse=None) | change
    c = cache()
    assert lib.ecospa_quant_cache_attn(ctx, C.byref(c), *a.values()) == code


def test_attention_asks_for_its_workspace(lib, ctx):
    big = cache(B=1, cap=100000, own_max=100000)
    need = lib.ecospa_quant_cache_attn_workspace_bytes(C.byref(big), 1)
    assert need > 0 and need % 256 == 0
    call = lambda: lib.ecospa_quant_cache_attn(ctx, C.byref(big), 1, 256, 256, None, 0, None, 512, 384, None)
    assert call() == B.ERR_WORKSPACE
    assert lib.ecospa_set_workspace(ctx, 1 << 20, need - 256) == B.OK
    assert call() == B.ERR_WORKSPACE
    assert lib.ecospa_quant_cache_attn_workspace_bytes(C.byref(cache(own_max=0)), 1) == 0
    assert lib.ecospa_quant_cache_attn_workspace_bytes(C.byref(cache()), 0) == 0


@pytest.mark.parametrize("change,code", [
    (dict(qkv=None), B.ERR_NULL), (dict(cos=1024), B.ERR_NULL), (dict(sin=1024), B.ERR_NULL), (dict(cos=1024, sin=2048, L_tab=9), B.ERR_NULL),
    (dict(pos=128, cos=1024, sin=2048, L_tab=9, q=None), B.ERR_NULL), (dict(pos=128, cos=1024, sin=2048), B.ERR_SHAPE),
    (dict(L=0), B.ERR_SHAPE), (dict(L=1 << 27), B.ERR_SHAPE), (dict(ld_qkv=568), B.ERR_SHAPE), (dict(ld_q=248), B.ERR_SHAPE),
    (dict(qkv=264), B.ERR_ALIGN), (dict(ld_qkv=580), B.ERR_ALIGN), (dict(q=520), B.ERR_ALIGN), (dict(ld_q=260), B.ERR_ALIGN),
    (dict(pos=128, cos=1028, sin=2048, L_tab=9), B.ERR_ALIGN),
], ids=str)
def test_append_refusals(lib, ctx, change, code):
    a = dict(L=2, qkv=256, ld_qkv=576, pos=None, cos=None, sin=None, L_tab=0, q=512, ld_q=256) | change
    c = cache()
    assert lib.ecospa_quant_cache_append(ctx, C.byref(c), *a.values()) == code


# ---- drawing tokens ----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("change,code", [
    (dict(logits=None), B.ERR_NULL), (dict(u=None), B.ERR_NULL), (dict(token=None), B.ERR_NULL), (dict(dtype=2), B.ERR_DTYPE),
    (dict(B=0), B.ERR_SHAPE), (dict(B=65536), B.ERR_SHAPE), (dict(V=0), B.ERR_SHAPE), (dict(V=(1 << 20) + 1, ld=1 << 21), B.ERR_SHAPE), (dict(ld=992), B.ERR_SHAPE),
    (dict(ld=1004), B.ERR_ALIGN), (dict(logits=264), B.ERR_ALIGN), (dict(u=514), B.ERR_ALIGN), (dict(top_k=1), B.ERR_ALIGN), (dict(prob=2), B.ERR_ALIGN),
    (dict(), B.ERR_WORKSPACE),
], ids=str)
def test_sample_refusals(lib, ctx, change, code):
    a = B.SampleArgs(*(dict(B=2, V=1000, dtype=B.BF16, logits=256, ld=1008, u=512, temperature=None, top_k=None, top_p=None, min_p=None, token=1024, prob=None) | change).values())
    assert lib.ecospa_sample(ctx, C.byref(a)) == code


def test_sample_without_arguments(lib, ctx):
    assert lib.ecospa_sample(ctx, None) == B.ERR_NULL
    assert lib.ecospa_sample(None, C.byref(B.SampleArgs())) == B.ERR_NULL
    assert lib.ecospa_sample_workspace_bytes(0, 10) == 0 and lib.ecospa_sample_workspace_bytes(1, (1 << 20) + 1) == 0
    need = lib.ecospa_sample_workspace_bytes(2, 1000)
    assert need > 0 and need % 256 == 0
    a = B.SampleArgs(2, 1000, B.BF16, 256, 1008, 512, None, None, None, None, 1024, None)
    assert lib.ecospa_set_workspace(ctx, 1 << 20, need - 256) == B.OK
    assert lib.ecospa_sample(ctx, C.byref(a)) == B.ERR_WORKSPACE
