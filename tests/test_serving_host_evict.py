"""Evictions whose outputs are inputs, or each other, are refused on the host, before anything is launched (no GPU needed: none of the addresses below
is ever read).  Rows would be overwritten while other wavefronts still read them."""
import ctypes as C

import pytest

from paper_2511_11641_amd import binding as B
from test_serving_host import cache, ctx, lib  # noqa: F401 (fixtures)

K, V, LENS, W, LENS_OUT, W_OUT, IDX = (1 << 20, 1 << 21, 1 << 22, 1 << 23, 1 << 24, 1 << 25, 1 << 26)
K_OUT, V_OUT = 1 << 27, 1 << 28


def call(lib, ctx, k_out=K_OUT, v_out=V_OUT, lens_out=LENS_OUT, w_out=W_OUT, idx=IDX, h=8):
    src, dst = cache(k=K, v=V, lens=LENS), cache(k=k_out, v=v_out, lens=None, cap=20, own_max=0, h=h)
    return lib.ecospa_cache_evict(ctx, C.byref(src), W, 10, 2, C.byref(dst), lens_out, w_out, idx)


SAME = [dict(k_out=K), dict(v_out=V), dict(k_out=V), dict(v_out=K), dict(k_out=K, v_out=V), dict(k_out=V_OUT), dict(lens_out=LENS), dict(w_out=W),
        dict(idx=LENS), dict(idx=W), dict(idx=LENS_OUT), dict(idx=W_OUT), dict(lens_out=W), dict(w_out=LENS), dict(w_out=LENS_OUT)]


@pytest.mark.parametrize("change", SAME, ids=[str(sorted(c)) + str(i) for i, c in enumerate(SAME)])
@pytest.mark.parametrize("listed", [True, False])
def test_outputs_that_are_inputs(lib, ctx, change, listed):  # noqa: F811
    if not listed:                                       # the list of rows in the workspace
        assert lib.ecospa_set_workspace(ctx, 1 << 30, 1 << 20) == B.OK
        if "idx" in change:
            return
        change = dict(change, idx=None)
    assert call(lib, ctx, **change) == B.ERR_SHAPE


def test_the_same_call_apart_is_not_refused(lib, ctx):  # noqa: F811
    assert call(lib, ctx, idx=None) == B.ERR_WORKSPACE   # no refusal of its arguments: the next one is for the memory that is missing


@pytest.mark.parametrize("h", [0, 6, 4, 8])
def test_the_query_heads_of_the_new_cache_play_no_part(lib, ctx, h):  # noqa: F811
    assert call(lib, ctx, idx=None, h=h) == B.ERR_WORKSPACE
