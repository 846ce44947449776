"""Serving entry points on the GPU against the fp64 oracle: lengths around the tiles, rows that see nothing, unequal kept widths,
grouped heads, strides, what lies in unused rows, streams, graphs.

Bounds.  bf16 has 8 significant bits, so rounding to nearest is off by at most 2^-8 of the value.  The attention output is a sum of p_j v_j with
p_j rounded to bf16 before the product and the sum rounded to bf16: |error| <= 2^-8 |o| + 2^-8 sum p |v|, and for fp32 exponentials and sums 2^-12 sum p |v|, for moved scores expm1(2 d) sum p |v|.
Scores are off by at most 128 roundings of their largest partial sum: d = 2^-17 sum |q k|; lse by that and its own rounding, the weights
by a factor of exp(2 d + lse's)."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2511_11641_amd import binding as B
from util import host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rnd(g, *shape, mul=1.0):
    return (mul * torch.randn(*shape, device="cuda", generator=g)).bfloat16()


class Case:
    """Caches, prefix and queries; rows beyond every length hold NaN."""

    def __init__(self, seed, Bn, L, h, h_kv, e, f, P, lens, cap=None, own_max=None, layout="heads", spread=1.0, scale=0.125):
        g = gen(seed)
        cap = max(max(lens), 1) + 3 if cap is None else cap
        if layout == "tokens":       # rows of all heads side by side, as a projection leaves them; prefix as columns of wider rows
            self.k, self.v = rnd(g, Bn, cap, h_kv, e).transpose(1, 2), rnd(g, Bn, cap, h_kv, f).transpose(1, 2)
            rows = rnd(g, max(P, 1), (h + h_kv) * e + h_kv * f)
            self.pk = rows[:P, h * e:(h + h_kv) * e].view(P, h_kv, e).transpose(0, 1)
            self.pv = rows[:P, (h + h_kv) * e:].view(P, h_kv, f).transpose(0, 1)
            self.q = rnd(g, Bn * L, h * e + 24, mul=spread)[:, 8:8 + h * e]
        else:
            self.k, self.v, self.pk, self.pv = rnd(g, Bn, h_kv, cap, e), rnd(g, Bn, h_kv, cap, f), rnd(g, h_kv, P, e), rnd(g, h_kv, P, f)
            self.q = rnd(g, Bn * L, h * e, mul=spread)
        dead = torch.arange(cap, device="cuda") >= torch.tensor([[max(n, 0)] for n in lens], device="cuda")
        self.k.masked_fill_(dead[:, None, :, None], float("nan"))
        self.v.masked_fill_(dead[:, None, :, None], float("nan"))
        self.w = torch.rand(Bn, h_kv, cap, device="cuda", generator=g)
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.B, self.L, self.h, self.h_kv, self.e, self.f, self.P, self.cap, self.scale = Bn, L, h, h_kv, e, f, P, cap, scale
        self.cache = B.KvCache(self.k, self.v, self.lens, h, scale, self.pk, self.pv, own_max=own_max)

    def run(self, ctx, lse=True, weights=True):
        o = torch.full((self.B * self.L, self.h * self.f), float("nan"), device="cuda", dtype=torch.bfloat16)
        ls = torch.full((self.B, self.h, self.L), float("nan"), device="cuda") if lse else None
        w = torch.full_like(self.w, -7.0) if weights else None
        ctx.ecospa_prefix_attn(self.cache, self.q, o, lse=ls, weights=self.w if weights else None, weights_out=w)
        return o, ls, w

    def check(self, o, lse=None, w=None):
        want = S.prefix_attn(host(self.q), host(self.k), host(self.v), self.lens.tolist(), self.h, self.scale, host(self.pk), host(self.pv), host(self.w))
        empty = np.isinf(want["lse"])
        d = 2.0 ** -17 * want["s_abs"] + 2.0 ** -21 * (1 + np.where(empty, 0, np.abs(want["lse"])))
        err = np.abs(host(o) - want["o"])
        moved = np.repeat(np.expm1(2 * d).transpose(0, 2, 1).reshape(self.B * self.L, self.h), self.f, axis=1)
        room = 2.0 ** -8 * np.abs(want["o"]) + (2.0 ** -8 + 2.0 ** -12 + moved) * want["av"]
        assert (err <= room).all(), f"o: {np.nanmax(err - room)} over at {np.argwhere(~(err <= room))[:3]}"
        if lse is not None:
            got = lse.double().cpu().numpy()
            assert np.array_equal(np.isneginf(got), empty)
            assert (np.abs(got[~empty] - want["lse"][~empty]) <= d[~empty]).all()
        if w is not None:
            got, alive = w.double().cpu().numpy(), np.arange(self.cap) < np.maximum(self.lens.cpu().numpy(), 0)[:, None, None]
            added = want["w"] - host(self.w)
            room = added * np.expm1(4 * d.max()) + 2.0 ** -20 * (want["w"] + 1e-3)
            assert (got[~np.broadcast_to(alive, got.shape)] == -7.0).all(), "entries beyond the lengths were written"
            assert (np.abs(got - want["w"])[np.broadcast_to(alive, got.shape)] <= room[np.broadcast_to(alive, got.shape)]).all()


LENGTHS = [
    # B, L, h, h_kv, P, lens
    (1, 1, 4, 4, 0, [1]), (1, 1, 4, 4, 0, [0]), (1, 1, 4, 2, 1, [0]), (1, 1, 6, 6, 61, [33]),
    (3, 1, 4, 4, 64, [0, 1, 65]), (3, 1, 4, 4, 63, [64, 63, 128]), (5, 1, 8, 1, 65, [31, 32, 33, 95, 97]), (2, 1, 32, 1, 130, [7, 260]),
    (4, 3, 4, 2, 0, [3, 1, 0, 70]), (2, 5, 6, 3, 129, [5, 66]), (3, 8, 8, 2, 40, [8, 40, 2]), (2, 40, 4, 2, 33, [40, 100]), (1, 70, 6, 2, 300, [170]),
    (2, 130, 4, 4, 0, [130, 129]), (3, 140, 12, 3, 20, [200, 140, 139]), (2, 97, 40, 1, 0, [97, 300]), (2, 15, 70, 2, 9, [15, 14]), (40, 1, 4, 2, 700, [1 + 13 * i % 97 for i in range(40)]), (9, 1, 16, 4, 2100, [1 + 301 * i % 1300 for i in range(9)]),
    (1, 1, 8, 8, 9000, [200]), (1, 2, 4, 4, 0, [20000]), (24, 2, 12, 3, 5000, [2 + 37 * i % 500 for i in range(24)]),
]


@pytest.mark.parametrize("Bn,L,h,h_kv,P,lens", LENGTHS)
def test_attention_over_lengths(ctx, Bn, L, h, h_kv, P, lens):
    c = Case(Bn + L, Bn, L, h, h_kv, 32, 32, P, lens)
    first = c.run(ctx)
    c.check(*first)
    again = c.run(ctx)
    assert all(torch.equal(x, y) for x, y in zip(first, again)), "not the same twice"


@pytest.mark.parametrize("e", [16, 32, 48, 64, 80, 128])
@pytest.mark.parametrize("f", [16, 48, 64, 96, 128])
def test_attention_over_widths(ctx, e, f):
    Case(e + f, 3, 1, 8, 4, e, f, 150, [40, 0, 111]).check(*Case(e + f, 3, 1, 8, 4, e, f, 150, [40, 0, 111]).run(ctx))
    c = Case(e * f, 2, 37, 8, 4, e, f, 90, [37, 61])          # more than 64 rows a request
    c.check(*c.run(ctx))
    c = Case(e - f, 33, 1, 8, 2, e, f, 1500, [1 + i for i in range(33)])      # requests put together on the prefix
    c.check(*c.run(ctx))


@pytest.mark.parametrize("P,lens,L", [(70, [40, 17, 5], 1), (1300, [3, 77, 200], 2), (0, [9, 70, 64], 4), (200, [50, 60, 70], 33)])
def test_attention_over_strides(ctx, P, lens, L):
    c = Case(5, 3, L, 6, 3, 48, 32, P, lens, layout="tokens")
    c.check(*c.run(ctx))
    o = torch.full((3 * L, 6 * 32 + 16), 5.0, device="cuda", dtype=torch.bfloat16)          # rows of a wider output
    ctx.ecospa_prefix_attn(c.cache, c.q, o[:, 8:8 + 192])
    assert (o[:, :8] == 5).all() and (o[:, 200:] == 5).all()
    c.check(o[:, 8:200])


def test_attention_optional_outputs_and_bounds(ctx):
    c = Case(6, 4, 2, 8, 2, 32, 64, 900, [30, 2, 0, 110])
    o, lse, w = c.run(ctx)
    o2, _, w2 = c.run(ctx, lse=False)
    assert torch.equal(o, o2) and torch.equal(w, w2)
    assert torch.equal(o, c.run(ctx, lse=False, weights=False)[0])
    w3 = c.w.clone()
    ctx.ecospa_prefix_attn(c.cache, c.q, o, weights=w3, weights_out=w3)          # in place
    alive = torch.arange(c.cap, device="cuda") < c.lens[:, None, None]
    assert torch.equal(torch.where(alive, w, c.w), w3)
    w4 = torch.zeros_like(w3)
    ctx.ecospa_prefix_attn(c.cache, c.q, o, weights_out=w4)                      # from nothing
    assert torch.allclose(torch.where(alive, w4 + c.w, c.w), w3, rtol=0, atol=1e-6)
    c.cache.own_max = 60                                                         # a length above the bound counts as the bound
    got = c.run(ctx)
    c.lens.clamp_(max=60)
    w60 = got[2].clone()
    w60[3, :, 60:] = -7.0
    c.check(got[0], got[1], w60)
    c.lens.fill_(-5)                                                             # and below zero as zero
    c.check(*c.run(ctx))


@pytest.mark.parametrize("spread", [0.0, 30.0, 300.0])
def test_attention_with_flat_and_steep_scores(ctx, spread):
    """Scores of up to several thousand: the running maximum moves, nothing overflows, and equal scores share evenly."""
    c = Case(7, 3, 1, 4, 2, 64, 64, 700, [5, 300, 64], spread=spread)
    c.check(*c.run(ctx))
    c = Case(8, 2, 20, 8, 2, 64, 32, 100, [130, 20], spread=spread)
    c.check(*c.run(ctx))


def test_attention_maxima_at_the_far_end(ctx):
    """Scores that grow along the keys move the reference in every tile; a huge last key takes everything."""
    c = Case(9, 2, 1, 2, 2, 32, 32, 500, [200, 90])
    ramp = torch.linspace(0, 60, 500, device="cuda")
    c.pk.copy_((c.q.view(2, 2, 32)[0].float() * 0.1)[:, None, :] * ramp[None, :, None])
    c.check(*c.run(ctx))
    c.k[0, :, 199] = 40 * c.q.view(2, 2, 32)[0]
    c.check(*c.run(ctx))


def test_attention_past_32_bits(ctx):
    """Rows 64 MB apart: offsets pass 2^31 elements inside one cache."""
    stride, n = (1 << 25) - 8, 70
    c = Case(10, 1, 1, 2, 1, 32, 32, 0, [n], cap=n)
    big = torch.empty(stride * n + 64, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.as_strided(big, (1, 1, n, 32), (0, 0, stride, 1), at) for at in (0, 32))
    k.copy_(c.k)
    v.copy_(c.v)
    c.cache = B.KvCache(k, v, c.lens, 2, c.scale)
    c.check(*c.run(ctx))
    ko = torch.zeros(1, 1, 64, 32, device="cuda", dtype=torch.bfloat16)
    vo, lens = torch.zeros_like(ko), torch.zeros(1, dtype=torch.int32, device="cuda")
    w = torch.arange(n, device="cuda", dtype=torch.float32).view(1, 1, n)
    ctx.ecospa_cache_evict(c.cache, w, 64, 0, ko, vo, lens)
    assert torch.equal(ko[0, 0], c.k[0, 0, 6:]) and torch.equal(vo[0, 0], c.v[0, 0, 6:]) and lens.item() == 64


@pytest.mark.parametrize("Bn,L,h,h_kv,e,f,P,lens,cap", [
    (3, 1, 8, 4, 48, 48, 100, [200, 33, 0], 50000), (2, 40, 4, 2, 48, 64, 77, [90, 40], 110000), (2, 1, 4, 2, 128, 96, 0, [70, 1], 60000),
    (1, 1, 4, 2, 48, 48, 262000, [10], 20), (5, 1, 4, 2, 64, 32, 262001, [10, 0, 3, 70, 1], 80), (4, 3, 4, 2, 96, 128, 110001, [3, 50, 9, 0], 60)])
def test_attention_of_large_caches(ctx, Bn, L, h, h_kv, e, f, P, lens, cap):
    """More than 96 MB of keys and values in own caches or in the prefix, each read by one item: loads that pass the caches by."""
    assert 2 * h_kv * (e + f) * max(Bn * cap, P) > 96e6
    c = Case(11, Bn, L, h, h_kv, e, f, P, lens, cap=cap)
    c.check(*c.run(ctx))


# ---- append -------------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("Bn,L,h,h_kv,e,f,cap,lens", [(1, 1, 1, 1, 16, 16, 1, [1]), (4, 1, 16, 16, 32, 32, 40, [1, 40, 7, 0]), (3, 5, 8, 2, 48, 128, 20, [5, 20, 3]),
                                                      (2, 70, 6, 3, 128, 64, 90, [70, 95]), (5, 1, 4, 4, 16, 80, 9, [9, 10, -1, 3, 1])])
def test_append(ctx, rope, Bn, L, h, h_kv, e, f, cap, lens):
    g = gen(Bn * L)
    qkv = rnd(g, Bn * L, (h + h_kv) * e + h_kv * f + 16)[:, :-16]
    k, v = rnd(g, Bn, h_kv, cap, e), rnd(g, Bn, h_kv, cap, f)
    w = torch.rand(Bn, h_kv, cap, device="cuda", generator=g)
    lens_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pos = torch.tensor([(11 * i) % 50 for i in range(Bn)], dtype=torch.int32, device="cuda")
    if rope:
        pos[-1] = 95                                     # some positions are outside the tables
        ang = torch.rand(h_kv, 100, e // 2, device="cuda", generator=g, dtype=torch.float64) * 100
        cos, sin = ang.cos().float(), ang.sin().float()
    args = (pos.tolist(), host(cos), host(sin)) if rope else (None, None, None)
    want = S.append(host(qkv), host(k), host(v), lens, h, *args, w=host(w))
    q = torch.full((Bn * L, h * e + 8), 3.0, device="cuda", dtype=torch.bfloat16)[:, :h * e]
    cache = B.KvCache(k, v, lens_d, h, 0.1)
    rows = qkv.clone()
    ctx.ecospa_cache_append(cache, qkv, pos if rope else None, rope=(cos, sin) if rope else None, q=q, weights=w)
    # a turned value is the sum of two products, each off by a rounding, and rounded to bf16
    big = 2.0 * np.abs(host(qkv)).max()
    for name, got, ref in (("q", q, want[0]), ("k", k, want[1])):
        assert (np.abs(host(got) - ref) <= (2.0 ** -8 * np.abs(ref) + 2.0 ** -22 * big if rope else 0.0)).all(), name
    assert np.array_equal(host(v), want[2]) and np.array_equal(host(w), want[3])
    if rope:                                             # in place on the rows of the projection
        k2 = k.clone()
        ctx.ecospa_cache_append(B.KvCache(k2, v, lens_d, h, 0.1), rows, pos, rope=(cos, sin), q=rows)
        assert torch.equal(rows[:, :h * e], q) and torch.equal(rows[:, h * e:], qkv[:, h * e:]) and torch.equal(k2, k)
    else:
        k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
        ctx.ecospa_cache_append(B.KvCache(k2, v2, lens_d, h, 0.1), qkv)
        assert torch.equal(k2[k2 != 0], k[k2 != 0]) and torch.equal(v2[v2 != 0], v[v2 != 0])


# ---- evict --------------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("Bn,h_kv,e,f,cap,lens,keep,recent", [
    (1, 1, 16, 16, 1, [1], 1, 0), (1, 2, 32, 48, 9, [9], 4, 4), (3, 2, 32, 32, 70, [0, 70, 65], 64, 10), (2, 3, 16, 128, 200, [200, 130], 129, 1),
    (4, 2, 48, 64, 1100, [1100, 1, 700, 699], 700, 333), (2, 2, 64, 64, 9000, [9000, 8500], 100, 50), (1, 1, 32, 32, 40000, [39999], 20000, 7),
    (2, 1, 32, 32, 50, [50, 20], 60, 60)])
@pytest.mark.parametrize("kind", ["spread", "ties", "values"])
def test_evict(ctx, Bn, h_kv, e, f, cap, lens, keep, recent, kind):
    g = gen(cap + keep)
    k, v = rnd(g, Bn, cap, h_kv, e).transpose(1, 2), rnd(g, Bn, h_kv, cap, f)
    w = torch.rand(Bn, h_kv, cap, device="cuda", generator=g)
    if kind == "ties":
        w = (w * 3).floor() * 0.25
    if kind == "values":
        pick = torch.rand(Bn, h_kv, cap, device="cuda", generator=g)
        for at, x in ((0.1, float("nan")), (0.2, float("inf")), (0.3, 0.0), (0.4, -0.0), (0.5, -float("inf")), (0.55, 3.4e38), (0.6, -1e-45)):
            w = torch.where((pick < at) & (pick >= at - 0.05), x, w)
    kept, new = S.evict(w.cpu().numpy(), lens, keep, recent)
    lens_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cap2 = keep + 2
    ko, vo = torch.full((Bn, h_kv, cap2, e), 9.0, device="cuda", dtype=torch.bfloat16), torch.full((Bn, h_kv, cap2, f), 9.0, device="cuda", dtype=torch.bfloat16)
    wo, lo = torch.full((Bn, h_kv, cap2), 9.0, device="cuda"), torch.full((Bn,), -9, dtype=torch.int32, device="cuda")
    idx = torch.full((Bn, h_kv, keep), -9, dtype=torch.int32, device="cuda")
    cache = B.KvCache(k, v, lens_d, h_kv, 0.1)
    ctx.ecospa_cache_evict(cache, w, keep, recent, ko, vo, lo, wo, idx)
    assert lo.tolist() == new
    for b in range(Bn):
        for hk in range(h_kv):
            r = torch.tensor(kept[b][hk], device="cuda", dtype=torch.long)
            n = len(r)
            assert torch.equal(idx[b, hk, :n].long(), r) and (idx[b, hk, n:] == -1).all()
            assert torch.equal(ko[b, hk, :n], k[b, hk, r]) and torch.equal(vo[b, hk, :n], v[b, hk, r])
            assert torch.equal(wo[b, hk, :n].view(torch.int32), w[b, hk, r].view(torch.int32))
            assert (ko[b, hk, n:] == 9).all() and (vo[b, hk, n:] == 9).all() and (wo[b, hk, n:] == 9).all()
    ko2, vo2, lo2 = torch.full_like(ko, 9.0), torch.full_like(vo, 9.0), torch.zeros_like(lo)
    ctx.ecospa_cache_evict(cache, w, keep, recent, ko2, vo2, lo2)          # the list in the workspace
    assert torch.equal(ko, ko2) and torch.equal(vo, vo2) and torch.equal(lo, lo2)


# ---- logits -------------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("V", [1, 7, 31, 33, 1000, 4096, 4097, 9001, 50257])
@pytest.mark.parametrize("dt,odt", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_logits(ctx, V, dt, odt):
    """Values that fp32 holds exactly at every step (multiples of 1/64 of limited size): results have to be equal, the best token too."""
    Bn, H, nb, nm = 5, 40, 9, 2
    rng = np.random.default_rng(V)
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    pitch = (V + 7) // 8 * 8 + 8
    x = rng.integers(-64, 65, (Bn, V)) / 8.0
    hist = rng.integers(-2, V + 2, (Bn, H)) if V > 50 else rng.integers(-1, V + 1, (Bn, H))
    hist[:, ::3] = hist[:, :1]                                          # repeated
    hl = np.array([H, 0, 17, H + 5, -1])
    rep, freq, pres, temp = np.array([1, 2, 4, 2, 0.5]), np.array([0, 0.25, 0.5, 1, 0.25]), np.array([0.5, 0, 0.25, 0, 1]), np.array([1, 2, 0.5, 4, 1])
    ids = rng.integers(-1, V + 1, (Bn, nb))
    ids[:, 5] = ids[:, 2]
    ids[:, 7] = ids[:, 2]                                               # listed three times
    bias = rng.integers(-8, 9, (Bn, nb)) / 4.0
    mask = rng.integers(0, 1 << 32, (nm, (V + 31) // 32 + 1), dtype=np.uint64).astype(np.uint32).view(np.int32)
    mask[1] = 0                                                         # nothing is allowed
    row = np.array([0, -1, 0, 1, 2])
    up = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()
    buf = torch.full((Bn, pitch), float("nan"), device="cuda", dtype=types[dt])
    buf[:, :V] = up(x, types[dt])
    out = torch.full((Bn, pitch), 77.0, device="cuda", dtype=types[odt])
    f32, i32 = torch.float32, torch.int32
    kw = dict(history=up(hist, i32), history_len=up(hl, i32), repetition=up(rep, f32), frequency=up(freq, f32), presence=up(pres, f32),
              temperature=up(temp, f32), bias_ids=up(ids, i32), bias=up(bias, f32), mask=up(mask, i32)[:, :(V + 31) // 32], mask_row=up(row, i32))
    ref = dict(history=hist, history_len=hl, repetition=rep, frequency=freq, presence=pres, temperature=temp, bias_ids=ids, bias=bias, mask=mask, mask_row=row)
    for drop in ((), ("mask", "mask_row"), ("history", "history_len"), ("bias", "bias_ids"), ("temperature", "repetition"), tuple(kw)):
        want, pick, lse = S.logits_process(x, **{n: y for n, y in ref.items() if n not in drop})
        got_pick, got_lse = ctx.ecospa_logits_process(buf[:, :V], out=out[:, :V], **{n: y for n, y in kw.items() if n not in drop})
        assert torch.equal(out[:, :V].cpu(), torch.from_numpy(want).float().to(types[odt])), drop
        assert (out[:, V:] == 77).all() and got_pick.tolist() == pick.tolist(), drop
        fine = np.isfinite(lse)
        got = got_lse.double().cpu().numpy()
        assert np.array_equal(got[~fine], lse[~fine]) and (np.abs(got[fine] - lse[fine]) <= 2.0 ** -19 * (2 + np.abs(lse[fine]))).all(), drop
    p2, l2 = ctx.ecospa_logits_process(buf[:, :V], **kw)                # without the processed logits; twice the same
    p3, l3 = ctx.ecospa_logits_process(buf[:, :V], out=buf[:, :V], **kw)      # in place
    assert torch.equal(p2, p3) and torch.equal(l2, l3)
    want = S.logits_process(x, **ref)[0]
    assert torch.equal(buf[:, :V].cpu(), torch.from_numpy(want).float().to(types[dt]))


@pytest.mark.parametrize("V", [16385, 20001, 32768])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_logits_of_many_rows(ctx, V, dt):
    """Rows for most of the chip, a vocabulary that one workgroup holds then: every row as the definition, exactly."""
    distinct, Bn, H = 5, 163, 900
    rng = np.random.default_rng(V)
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dt]
    of = np.arange(Bn) % distinct
    x = rng.integers(-64, 65, (distinct, V)) / 8.0
    x[1, [V - 1, V - 7]] = 20.0                                         # the lower of equal ones, in the last chunk
    hist = rng.integers(0, V, (distinct, H))
    hist[1] %= V - 7
    hist[:, ::3] = hist[:, :1]
    ids = np.stack([rng.choice(V, 9, replace=False) for _ in range(distinct)])
    ids[1] %= V - 7
    ids[:, 7] = ids[:, 2]
    mask = rng.integers(0, 1 << 32, (2, (V + 31) // 32), dtype=np.uint64).astype(np.uint32).view(np.int32)
    mask[1] = 0
    ref = dict(history=hist, repetition=np.array([1, 2, 4, 2, 0.5]), frequency=np.array([0, 0.25, 0.5, 1, 0.25]), presence=np.array([0.5, 0, 0.25, 0, 1]),
               temperature=np.array([1, 2, 0.5, 4, 1]), bias_ids=ids, bias=rng.integers(-8, 9, (distinct, 9)) / 4.0, mask=mask, mask_row=np.array([0, -1, 0, 1, 2]))
    want, pick, lse = S.logits_process(x, **ref)
    up = lambda n, a: torch.from_numpy(np.ascontiguousarray(a if n == "mask" else a[of])).to(torch.int32 if a.dtype.kind == "i" and n != "temperature" else torch.float32).cuda()
    buf = torch.full((Bn, (V + 7) // 8 * 8 + 8), float("nan"), device="cuda", dtype=t)
    buf[:, :V] = torch.from_numpy(x[of]).to(t).cuda()
    out = torch.full_like(buf, 77.0)
    got_pick, got_lse = ctx.ecospa_logits_process(buf[:, :V], out=out[:, :V], **{n: up(n, a) for n, a in ref.items()})
    assert torch.equal(out[:, :V].cpu(), torch.from_numpy(want[of]).float().to(t)) and (out[:, V:] == 77).all()
    assert got_pick.tolist() == pick[of].tolist() and pick[1] == V - 7
    got, lse = got_lse.double().cpu().numpy(), lse[of]
    fine = np.isfinite(lse)
    assert np.array_equal(got[~fine], lse[~fine]) and (np.abs(got[fine] - lse[fine]) <= 2.0 ** -19 * (2 + np.abs(lse[fine]))).all()


def test_logits_values_and_ties(ctx):
    V = 9000
    x = torch.zeros(6, V, device="cuda")
    x[0, [4500, 8000]] = 3.0                             # the lower of equal ones, in different workgroups
    x[1] = -float("inf")
    x[2] = float("nan")
    x[3, 10], x[3, 20] = float("nan"), 1.0
    x[4, 7777] = float("inf")
    x[5] = -3.4e38
    pick, lse = ctx.ecospa_logits_process(x)
    assert pick.tolist() == [4500, -1, -1, 20, 7777, 0]
    assert lse[1].item() == -float("inf") and torch.isnan(lse[2]) and torch.isnan(lse[3]) and lse[4].item() == float("inf")
    assert abs(lse[0].item() - np.log(2 * np.exp(3.0) + V - 2)) < 1e-5 and abs(lse[5].item() + 3.4e38) < 1e33


def test_logits_long_history(ctx):
    """Counts of thousands of one token, spread over the whole history."""
    V, H = 70001, 60000
    g = gen(3)
    hist = torch.randint(0, V, (2, H), device="cuda", generator=g, dtype=torch.int32)
    hist[0, ::2] = 69999
    x, out = (torch.zeros(2, (V + 7) // 8 * 8, device="cuda")[:, :V] for _ in range(2))
    ctx.ecospa_logits_process(x, out=out, history=hist, frequency=torch.full((2,), 0.5, device="cuda"))
    for b in range(2):
        assert torch.equal(out[b], -0.5 * torch.bincount(hist[b].long(), minlength=V).float())


# ---- streams and graphs -------------------------------------------------------------------------------------------------------------------
def _decode(ctx, st):
    ctx.ecospa_cache_append(st["cache"], st["qkv"], st["pos"], rope=st["rope"], q=st["q"], weights=st["w"])
    ctx.ecospa_prefix_attn(st["cache"], st["q"], st["o"], lse=st["lse"], weights=st["w"], weights_out=st["w"])
    ctx.ecospa_cache_evict(st["cache"], st["w"], 24, 8, st["ko"], st["vo"], st["lens2"], st["w2"], st["idx"])
    ctx.ecospa_logits_process(st["logits"], out=st["out"], history=st["hist"], repetition=st["rep"], pick=st["pick"], lse=st["llse"])


def _state(seed, Bn=6, h=8, h_kv=4, e=32, f=48, P=1900, cap=64):
    g = gen(seed)
    k, v = rnd(g, Bn, h_kv, cap, e), rnd(g, Bn, h_kv, cap, f)
    lens = torch.randint(1, cap + 1, (Bn,), device="cuda", generator=g, dtype=torch.int32)
    ang = torch.rand(h_kv, 4000, e // 2, device="cuda", generator=g) * 50
    z = lambda *s, **kw: torch.zeros(*s, device="cuda", **kw)
    i32, bf = dict(dtype=torch.int32), dict(dtype=torch.bfloat16)
    return dict(cache=B.KvCache(k, v, lens, h, 0.15, rnd(g, h_kv, P, e), rnd(g, h_kv, P, f)), qkv=rnd(g, Bn, (h + h_kv) * e + h_kv * f),
                pos=(lens + P).int(), rope=(ang.cos(), ang.sin()), q=z(Bn, h * e, **bf), w=torch.rand(Bn, h_kv, cap, device="cuda", generator=g),
                o=z(Bn, h * f, **bf), lse=z(Bn, h, 1), ko=z(Bn, h_kv, 24, e, **bf), vo=z(Bn, h_kv, 24, f, **bf), lens2=z(Bn, **i32), w2=z(Bn, h_kv, 24),
                idx=z(Bn, h_kv, 24, **i32), logits=rnd(g, Bn, 12000), out=z(Bn, 12000, **bf), hist=torch.randint(0, 12000, (Bn, 50), device="cuda", generator=g, **i32),
                rep=torch.full((Bn,), 1.3, device="cuda"), pick=z(Bn, **i32), llse=z(Bn))


OUT = ("q", "w", "o", "lse", "ko", "vo", "lens2", "w2", "idx", "out", "pick", "llse")


def test_another_stream(ctx):
    a, b = _state(1), _state(1)
    _decode(ctx, a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    other = B.Context("cuda:0", stream=s)
    with torch.cuda.stream(s):
        _decode(other, b)
    s.synchronize()
    assert all(torch.equal(a[n], b[n]) for n in OUT) and torch.equal(a["cache"].k, b["cache"].k)


def test_a_decoding_step_in_a_graph():
    """Recorded once, replayed with new inputs in the same buffers and eager work in between: every replay as the eager calls."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = B.Context("cuda:0", stream=s)
        st = _state(2)
        _decode(ctx, st)                                  # the workspace grows outside the recording
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            _decode(ctx, st)
        for seed in (3, 4, 5):
            new, eager = _state(seed), _state(seed)
            for n in ("qkv", "pos", "w", "logits", "hist", "rep"):
                st[n].copy_(new[n])
            for n in ("k", "v", "lens", "pk", "pv"):
                getattr(st["cache"], n).copy_(getattr(new["cache"], n))
            st["rope"][0].copy_(new["rope"][0])
            st["rope"][1].copy_(new["rope"][1])
            for n in ("ko", "vo", "w2"):                  # rows behind a short cache's last one are not written
                st[n].zero_()
            graph.replay()
            _decode(ctx, eager)
            s.synchronize()
            assert all(torch.equal(st[n], eager[n]) for n in OUT) and torch.equal(st["cache"].k, eager["cache"].k)
