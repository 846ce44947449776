"""Attention over a shared prefix with queries and live keys that are not numbers: a row that meets one has an output, a log-sum-exp and weights that
are not numbers either, however the call is cut; every other row, and what a row does not see, is as if it were not there.  Bounds of finite values:
see test_gpu_serving.py."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2511_11641_amd import binding as B
from test_gpu_serving import Case, ctx  # noqa: F401 (ctx: the fixture)
from test_prefix_attn_cuts import FIELDS
from util import host

pytestmark = pytest.mark.gpu


def cut(c, weights):
    out = (C.c_int * 32)()
    n = B.load()._Z15prefix_attn_cutRK12ecospa_cacheiiPi(c.cache._ref, c.L, int(weights), out)
    return dict(zip(FIELDS, out[:n]))


def check(c, o, lse, w):
    with np.errstate(all="ignore"):
        want = S.prefix_attn(host(c.q), host(c.k), host(c.v), c.lens.tolist(), c.h, c.scale, host(c.pk), host(c.pv), host(c.w))
        empty = np.isneginf(want["lse"])
        d = 2.0 ** -17 * want["s_abs"] + 2.0 ** -21 * (1 + np.where(empty, 0, np.abs(want["lse"])))
        moved = np.repeat(np.expm1(2 * d).transpose(0, 2, 1).reshape(c.B * c.L, c.h), c.f, axis=1)
        got_o, got_lse, got_w = host(o), lse.double().cpu().numpy(), w.double().cpu().numpy()
        room_o = 2.0 ** -8 * np.abs(want["o"]) + (2.0 ** -8 + 2.0 ** -12 + moved) * want["av"]
        room_w = (want["w"] - host(c.w)) * np.expm1(4 * np.where(np.isfinite(d), d, 0).max()) + 2.0 ** -20 * (want["w"] + 1e-3)
        alive = np.broadcast_to(np.arange(c.cap) < np.maximum(c.lens.cpu().numpy(), 0)[:, None, None], got_w.shape)
        for name, got, ref, room in (("o", got_o, want["o"], room_o), ("lse", got_lse, want["lse"], np.where(empty, 0, d)),
                                     ("w", np.where(alive, got_w, 0), np.where(alive, want["w"], 0), room_w)):
            nan = np.isnan(ref)
            assert np.array_equal(np.isnan(got), nan), f"{name}: not a number in {np.isnan(got).sum()} places instead of {nan.sum()}, first {np.argwhere(np.isnan(got) != nan)[:3]}"
            assert np.array_equal(np.isinf(got), np.isinf(ref)), name
            fine = np.isfinite(ref)
            assert (np.abs(got - ref)[fine] <= room[fine]).all(), name
        assert (got_w[~alive] == -7.0).all()
    return want


# how the call is cut: items that are the whole row or pieces of it, joined by a row's own threads or a workgroup; scores kept for the weights or not
SHAPES = {
    "whole": (3, 2, 4, 2, 32, 32, 40, [9, 30, 17]),
    "whole, many rows": (2, 40, 4, 2, 32, 48, 33, [40, 70]),
    "whole, scores read again": (2, 9, 4, 2, 16, 32, 20, [40, 25]),
    "few pieces": (1, 2, 4, 4, 32, 32, 1500, [40]),
    "few pieces, keys of a wide head": (2, 1, 4, 2, 128, 96, 700, [200, 33]),
    "many pieces": (3, 1, 4, 4, 32, 32, 5000, [20, 1, 7]),
    "many pieces, shared rows": (40, 1, 4, 2, 48, 64, 2100, [1 + 5 * i % 33 for i in range(40)]),
    "pieces, scores read again": (3, 9, 6, 2, 32, 32, 2100, [90, 9, 70]),
    "pieces, many rows": (1, 70, 4, 2, 64, 64, 300, [170]),
    "nothing but own keys": (2, 3, 4, 2, 32, 32, 0, [70, 2]),
}


def test_the_shapes_are_cut_as_they_say(ctx):
    cuts = {n: cut(Case(1, *s), True) for n, s in SHAPES.items()}
    assert {n for n, a in cuts.items() if a["slots"] == 0} >= {"whole", "whole, many rows", "whole, scores read again"}
    pieces = {n: a["slots"] for n, a in cuts.items() if a["slots"]}
    assert any(x <= 4 for x in pieces.values()) and any(x > 16 for x in pieces.values())
    assert {(bool(a["slots"]), bool(a["keep"])) for a in cuts.values()} == {(x, y) for x in (False, True) for y in (False, True)}
    assert {a["joint"] for a in cuts.values()} == {0, 1}


@pytest.mark.parametrize("shape", SHAPES)
def test_queries_that_are_not_numbers(ctx, shape):
    c = Case(21, *SHAPES[shape])
    b, t, i = c.B - 1, c.L // 2, 1
    c.q.view(c.B, c.L, c.h, c.e)[b, t, i, 5] = float("nan")
    want = check(c, *c.run(ctx))
    seen = c.P + max(int(c.lens[b]) - c.L + 1 + t, 0)
    assert np.isnan(want["lse"][b, i, t]) == (seen > 0) and np.isnan(want["lse"]).sum() == (seen > 0)


@pytest.mark.parametrize("shape,where", [(n, x) for n, s in SHAPES.items() for x in ("prefix", "own", "newest") if s[6] or x != "prefix"])
@pytest.mark.parametrize("value", ["nan", "inf"])
def test_keys_that_are_not_numbers(ctx, shape, value, where):
    c = Case(22, *SHAPES[shape])
    c.q.view(-1, c.e)[:, 2].abs_().clamp_(min=0.125)            # a key of +inf there has a score of +inf
    b, hk = c.B - 1, c.h_kv - 1
    if where == "prefix":
        c.pk[hk, c.P // 2, 2] = float(value)
    else:
        c.k[b, hk, 0 if where == "own" else int(c.lens[b]) - 1, 2] = float(value)      # earlier queries of the request do not see the newest one
    want = check(c, *c.run(ctx))
    assert np.isnan(want["lse"]).any() and np.isfinite(want["lse"]).any() and np.isnan(want["w"]).any()


@pytest.mark.parametrize("shape", ["many pieces", "pieces, many rows", "whole"])
def test_every_query_is_not_a_number(ctx, shape):
    c = Case(23, *SHAPES[shape])
    c.q.fill_(float("nan"))
    check(c, *c.run(ctx))
