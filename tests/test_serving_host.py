"""Refusals of the serving entry points: every argument is looked at on the host before anything is launched (no GPU needed:
none of the addresses below is ever read)."""
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
    c = B.Cache(B.BF16, 2, 8, 4, 32, 48, 100, 90, 64, 0.125, 4096, 8192, 4 * 100 * 32, 100 * 32, 32, 4 * 100 * 48, 100 * 48, 48,
                16384, 32768, 64 * 32, 32, 64 * 48, 48, 65536)
    for n, x in kw.items():
        setattr(c, n, x)
    return c


BAD_CACHES = [
    (dict(k=None), B.ERR_NULL), (dict(v=None), B.ERR_NULL), (dict(lens=None), B.ERR_NULL), (dict(pk=None), B.ERR_NULL), (dict(pv=None), B.ERR_NULL),
    (dict(dtype=B.F32), B.ERR_DTYPE), (dict(dtype=7), B.ERR_DTYPE),
    (dict(B=0), B.ERR_SHAPE), (dict(h=0), B.ERR_SHAPE), (dict(h=6), B.ERR_SHAPE), (dict(h_kv=0), B.ERR_SHAPE), (dict(h=2), B.ERR_SHAPE),
    (dict(cap=0, own_max=0), B.ERR_SHAPE), (dict(own_max=101), B.ERR_SHAPE), (dict(own_max=-1), B.ERR_SHAPE), (dict(P=-1), B.ERR_SHAPE),
    (dict(kp_qk=24), B.ERR_SHAPE), (dict(kp_qk=0), B.ERR_SHAPE), (dict(kp_vo=144, v_st=144), B.ERR_SHAPE), (dict(kp_vo=8), B.ERR_SHAPE),
    (dict(scale=0.0), B.ERR_SHAPE), (dict(scale=-1.0), B.ERR_SHAPE), (dict(scale=float("nan")), B.ERR_SHAPE), (dict(scale=float("inf")), B.ERR_SHAPE),
    (dict(k_st=24), B.ERR_SHAPE), (dict(v_st=40), B.ERR_SHAPE), (dict(pk_st=16), B.ERR_SHAPE), (dict(pv_st=1 << 25), B.ERR_SHAPE),
    (dict(k_st=1 << 25), B.ERR_SHAPE), (dict(k_sb=-8), B.ERR_SHAPE), (dict(pv_sh=-8), B.ERR_SHAPE),
    (dict(k=4104), B.ERR_ALIGN), (dict(pv=32776), B.ERR_ALIGN), (dict(k_st=36), B.ERR_ALIGN), (dict(v_sb=4), B.ERR_ALIGN), (dict(pk_sh=2052), B.ERR_ALIGN),
    (dict(B=40000), B.ERR_SHAPE),
]


@pytest.mark.parametrize("change,code", BAD_CACHES, ids=[str(c) for c, _ in BAD_CACHES])
def test_caches_are_refused(lib, ctx, change, code):
    c = cache(**change)
    assert lib.ecospa_prefix_attn(ctx, C.byref(c), 1, 256, 256, 512, 384, None, None, None) == code
    assert lib.ecospa_prefix_attn_workspace_bytes(C.byref(c), 1, 1) == 0
    assert lib.ecospa_cache_append(ctx, C.byref(c), 1, 256, 576, None, None, None, 0, 512, 256, None) == code
    if not {"pk", "pv", "P", "pk_st", "pv_st", "pk_sh", "pv_sh"} & set(change):
        assert lib.ecospa_cache_evict(ctx, C.byref(c), 256, 10, 2, C.byref(cache()), 512, None, 1024) == code


def test_attention_refusals(lib, ctx):
    c = cache()

    def call(q=256, ld_q=256, o=512, ld_o=384, L=1, lse=None, w_in=None, w_out=None, desc=c, x=ctx):
        return lib.ecospa_prefix_attn(x, C.byref(desc) if desc else None, L, q, ld_q, o, ld_o, lse, w_in, w_out)

    assert call(x=None) == call(desc=None) == call(q=None) == call(o=None) == call(w_in=256) == B.ERR_NULL
    assert call(L=0) == call(ld_q=248) == call(ld_o=376) == call(L=1 << 27) == B.ERR_SHAPE
    assert call(q=264) == call(o=520) == call(ld_q=260) == call(ld_o=388) == B.ERR_ALIGN
    # pieces of a long prefix are joined in the workspace: none attached
    long = cache(P=1 << 16)
    need = lib.ecospa_prefix_attn_workspace_bytes(C.byref(long), 1, 0)
    assert need > 0 and call(desc=long) == B.ERR_WORKSPACE
    assert lib.ecospa_set_workspace(ctx, 1 << 20, 256) == B.OK and call(desc=long) == B.ERR_WORKSPACE
    # weights without lse keep their row statistics there
    assert lib.ecospa_set_workspace(ctx, None, 0) == B.OK and call(w_out=256) == B.ERR_WORKSPACE


def test_append_refusals(lib, ctx):
    c = cache()

    def call(qkv=256, ld=576, pos=None, cos=None, sin=None, tab=0, q=None, ld_q=0, L=1, x=ctx, desc=c):
        return lib.ecospa_cache_append(x, C.byref(desc) if desc else None, L, qkv, ld, pos, cos, sin, tab, q, ld_q, None)

    assert call(x=None) == call(desc=None) == call(qkv=None) == B.ERR_NULL
    rope = dict(pos=256, cos=512, sin=1024, tab=64, q=2048, ld_q=256)
    assert call(**dict(rope, sin=None)) == call(**dict(rope, pos=None)) == call(**dict(rope, q=None)) == B.ERR_NULL
    assert call(L=0) == call(ld=568) == call(**dict(rope, tab=0)) == call(**dict(rope, ld_q=248)) == B.ERR_SHAPE
    assert call(qkv=264) == call(ld=580) == call(**dict(rope, q=2056)) == call(**dict(rope, cos=520)) == B.ERR_ALIGN


def test_evict_refusals(lib, ctx):
    src, dst = cache(), cache(cap=20, own_max=0)

    def call(keep=10, recent=2, w=256, d=dst, lens=512, idx=1024, s=src, x=ctx):
        return lib.ecospa_cache_evict(x, C.byref(s) if s else None, w, keep, recent, C.byref(d) if d else None, lens, None, idx)

    assert call(x=None) == call(s=None) == call(d=None) == call(w=None) == call(lens=None) == call(d=cache(k=None)) == B.ERR_NULL
    assert call(keep=0) == call(recent=-1) == call(recent=11) == call(keep=21) == B.ERR_K
    assert call(d=cache(B=3)) == call(d=cache(h_kv=2)) == call(d=cache(kp_vo=32)) == B.ERR_SHAPE
    assert call(d=cache(v=8200)) == B.ERR_ALIGN
    assert call(idx=None) == B.ERR_WORKSPACE


def test_evict_refuses_its_inputs_as_outputs(lib, ctx):
    src, dst = cache(lens=4096), cache(cap=20, own_max=0)
    call = lambda lens, w_out: lib.ecospa_cache_evict(ctx, C.byref(src), 256, 10, 2, C.byref(dst), lens, w_out, None)
    assert call(4096, None) == call(512, 256) == B.ERR_SHAPE
    assert call(512, 768) == B.ERR_WORKSPACE


def test_logits_refusals(lib, ctx):
    def call(x=ctx, **kw):
        q = B.Logits(2, 100, B.BF16, B.BF16, 256, 512, 104, 104, None, None, 0, 0, None, None, None, None, None, None, None, None, 0, 0, 1024, 2048)
        for n, y in kw.items():
            setattr(q, n, y)
        return lib.ecospa_logits_process(x, C.byref(q))

    assert call(x=None) == call(logits=None) == call(out=None, pick=None, lse=None) == B.ERR_NULL
    assert lib.ecospa_logits_process(ctx, None) == B.ERR_NULL
    assert call(n_bias=2) == call(n_bias=2, bias=256) == call(mask=256, n_masks=1, ld_mask=4) == B.ERR_NULL
    assert call(dtype=2) == call(out_dtype=5) == B.ERR_DTYPE
    assert call(B=0) == call(V=0) == call(B=65536) == call(V=(1 << 24) + 1, ld=1 << 25, ld_out=1 << 25) == call(ld=96) == call(ld_out=96) == B.ERR_SHAPE
    assert call(n_bias=-1) == call(n_bias=1024, bias=256, bias_ids=256) == call(history=256, ld_history=1 << 22) == B.ERR_SHAPE
    assert call(mask=256, mask_row=256, n_masks=0, ld_mask=4) == call(mask=256, mask_row=256, n_masks=1, ld_mask=3) == B.ERR_SHAPE
    assert call(logits=264) == call(out=520) == call(ld=108) == call(ld_out=108) == B.ERR_ALIGN
    assert lib.ecospa_logits_workspace_bytes(2, 100) == 0 and lib.ecospa_logits_workspace_bytes(0, 100) == 0
    need = lib.ecospa_logits_workspace_bytes(1, 200000)
    assert need > 0 and call(B=1, V=200000, ld=200000, ld_out=200000) == B.ERR_WORKSPACE
