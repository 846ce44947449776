"""Caches of 8-bit floats on the GPU against the fp64 oracle: what an append leaves in codes and scales, attention over lengths around the tiles,
pieces and blocks, rows that see nothing, unequal kept widths, grouped heads, strides, what lies in unused rows, results joined in.

Bounds.  Codes and scales are compared exactly, given the keys as the library turned them: those are read back from caches of bf16 that the same rows
go into.  The attention output is a sum of p_j v_j with p_j (times its scale, a power of two) rounded to bf16, off by 2^-8 of it at most, and the sum rounded to bf16:
|error| <= 2^-8 |o| + 2^-8 sum p |v|, and for fp32 exponentials and sums 2^-12 sum p |v|, for moved scores expm1(2 d) sum p |v|.  Scores are off by at
most 128 roundings of their largest partial sum: d = 2^-17 sum |q k|; lse by that and its own rounding."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2511_11641_amd import binding as B
from util import host

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rnd(g, *shape, mul=1.0):
    return (mul * torch.randn(*shape, device="cuda", generator=g)).bfloat16()


def values(t):
    return t.float().cpu().numpy().astype(np.float64)


class Caches:
    """Caches of random codes and scales; rows beyond every length hold NaN, scales of blocks without a row too."""

    def __init__(self, seed, Bn, h, h_kv, e, f, lens, block, cap=None, layout="heads", own_max=None, scale=0.125, powers=True, shared=False):
        g = gen(seed)
        self.cap = cap = max(max(lens), 1) + 3 if cap is None else cap
        codes = lambda d: (torch.randn(Bn, h_kv, cap, d, device="cuda", generator=g) * 40).clamp(-448, 448).to(F8)
        if layout == "tokens":      # rows of all heads side by side, with room behind them
            self.k = codes(e).transpose(1, 2).contiguous().transpose(1, 2)
            wide = torch.zeros(Bn, cap, h_kv, f + 16, dtype=torch.uint8, device="cuda")
            wide[..., :f] = codes(f).transpose(1, 2).view(torch.uint8)
            self.v = wide.view(F8)[..., :f].transpose(1, 2)
        elif shared:                # one head's rows for all
            one = lambda d: (torch.randn(1, 1, cap, d, device="cuda", generator=g) * 40).clamp(-448, 448).to(F8).view(torch.uint8)
            k, v = one(e), one(f)
            for t in (k, v):
                t[:, :, max(lens):] = 0x7f
            self.k, self.v = k.view(F8).expand(Bn, h_kv, cap, e), v.view(F8).expand(Bn, h_kv, cap, f)
        else:
            self.k, self.v = codes(e), codes(f)
        n = (cap + block - 1) // block
        scales = lambda: torch.ldexp(torch.ones(Bn, h_kv, n, device="cuda"), torch.randint(-7, -3, (Bn, h_kv, n), device="cuda", generator=g)) * (
            1.0 if powers else 1.0 + torch.rand(Bn, h_kv, n, device="cuda", generator=g))
        self.k_scale, self.v_scale = scales(), scales()
        at = torch.tensor([[max(x, 0)] for x in lens], device="cuda")
        dead = torch.arange(cap, device="cuda") >= at
        for t in () if shared else (self.k, self.v):
            t.view(torch.uint8).masked_fill_(dead[:, None, :, None], 0x7f)
        unused = torch.arange(n, device="cuda") * block >= at
        self.k_scale.masked_fill_(unused[:, None], float("nan"))
        self.v_scale.masked_fill_(unused[:, None], float("nan"))
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.B, self.h, self.h_kv, self.e, self.f, self.block, self.scale = Bn, h, h_kv, e, f, block, scale
        self.own_max, self.shared = own_max, shared
        self.cache = B.QuantCache(self.k, self.v, self.k_scale, self.v_scale, self.lens, h, scale, block, own_max=own_max)

    def host(self):
        n = int(self.lens.max()) if self.shared else self.cap
        return {"k": values(self.k[:, :, :n]), "v": values(self.v[:, :, :n]), "k_scale": values(self.k_scale), "v_scale": values(self.v_scale)}


def attend(ctx, c, L, seed, prior=False, spread=1.0):
    g = gen(seed)
    q = rnd(g, c.B * L, c.h * c.e + 24, mul=spread)[:, 8:8 + c.h * c.e]
    wide = torch.full((c.B * L, c.h * c.f + 8), 3.0, device="cuda", dtype=torch.bfloat16)
    o, lse = wide[:, :c.h * c.f], torch.full((c.B, c.h, L), float("nan"), device="cuda")
    o_in = lse_in = None
    if prior:
        o_in, lse_in = rnd(g, c.B * L, c.h * c.f), 3.0 * torch.randn(c.B, c.h, L, device="cuda", generator=g)
        hole = torch.rand(c.B, c.h, L, device="cuda", generator=g) < 0.2
        lse_in.masked_fill_(hole, float("-inf"))      # nothing in front: what lies in o_in plays no part
        o_in.view(c.B, L, c.h, c.f).masked_fill_(hole.transpose(1, 2)[..., None], float("nan"))
    ctx.ecospa_quant_cache_attn(c.cache, q, o, lse=lse, o_in=o_in, lse_in=lse_in)
    assert bool((wide[:, c.h * c.f:] == 3.0).all())
    lens = np.clip(c.lens.cpu().numpy(), 0, c.cap if c.own_max is None else c.own_max)
    want = Q.attn(host(q), c.host(), lens, c.h, c.scale, c.block, None if o_in is None else host(o_in), None if lse_in is None else lse_in.double().cpu().numpy())
    empty = np.isinf(want["lse"])
    d = 2.0 ** -17 * want["s_abs"] + 2.0 ** -21 * (1 + np.where(empty, 0, np.abs(want["lse"])))
    moved = np.repeat(np.expm1(2 * d).transpose(0, 2, 1).reshape(c.B * L, c.h), c.f, axis=1)
    room = 2.0 ** -8 * np.abs(want["o"]) + (2.0 ** -8 + 2.0 ** -12 + moved) * want["av"]
    err = np.abs(host(o) - want["o"])
    assert (err <= room).all(), f"o: {np.nanmax(err - room)} over at {np.argwhere(~(err <= room))[:3]}"
    got = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(got), empty)
    assert (np.abs(got[~empty] - want["lse"][~empty]) <= d[~empty]).all()


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("L", [1, 2, 7])
def test_lengths_around_tiles_and_blocks(ctx, L, block):
    lens = [0, 1, 2, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]
    attend(ctx, Caches(L * block, len(lens), 4, 2, 32, 32, lens, block), L, 1)


@pytest.mark.parametrize("e,f", [(16, 16), (32, 64), (48, 112), (64, 48), (80, 128), (96, 32), (112, 80), (128, 96)])
@pytest.mark.parametrize("h,h_kv,L", [(3, 3, 1), (8, 2, 3), (6, 1, 5), (4, 1, 40)])
def test_widths_and_groups(ctx, e, f, h, h_kv, L):
    attend(ctx, Caches(e + f + L, 3, h, h_kv, e, f, [70, 0, 41], 16, layout="tokens" if L % 2 else "heads"), L, 2, prior=L == 3)


@pytest.mark.parametrize("rows", [15, 16, 17, 31, 32, 33, 63, 64, 65, 150])
def test_rows_around_the_tiles(ctx, rows):
    attend(ctx, Caches(rows, 2, 1, 1, 32, 48, [rows + 40, rows - 3], 32), rows, 3)


@pytest.mark.parametrize("n", [255, 256, 257, 3000, 9001])
@pytest.mark.parametrize("prior", [False, True])
def test_pieces(ctx, n, prior):
    attend(ctx, Caches(n, 2, 4, 2, 64, 64, [n, n // 3], 64), 1, 4, prior)
    attend(ctx, Caches(n, 1, 2, 1, 96, 128, [n], 16), 3, 5, prior)


WIDTHS = [(16, 32), (32, 48), (32, 112), (48, 16), (64, 64), (64, 128), (80, 32), (96, 64), (96, 96), (128, 32), (112, 48), (128, 128)]      # of every kernel: 32-dim steps of a key, dims of a value a lane holds


@pytest.mark.parametrize("e,f", WIDTHS)
@pytest.mark.parametrize("g,L", [(2, 10), (3, 15), (1, 70)])
def test_many_rows_of_many_heads(ctx, e, f, g, L):
    """Enough workgroups for tiles of 32 and 64 queries a wavefront, the last one not full."""
    attend(ctx, Caches(e + f, 4, 128 * g, 128, e, f, [75, 2, 40, 33], 16), L, 9, prior=g == 2)


@pytest.mark.parametrize("e,f", WIDTHS)
@pytest.mark.parametrize("L", [1, 3])
def test_caches_beyond_the_last_level_cache(ctx, e, f, L):
    """More than 256 MB by strides and bound: all heads of all requests in the same memory."""
    Bn, h_kv, lens = 2, 32, [300, 41]
    c = Caches(e + f, Bn, h_kv, h_kv, e, f, lens, 64, cap=((1 << 28) // (Bn * h_kv * (e + f)) + 64) // 64 * 64 + 64, shared=True)
    assert Bn * h_kv * c.cap * (e + f) > 1 << 28
    attend(ctx, c, L, 10)


def test_scales_that_are_no_powers_of_two(ctx):
    c = Caches(3, 2, 4, 2, 64, 64, [300, 77], 32, powers=False)
    # a probability times such a scale is rounded as any other product: the bound is the same
    attend(ctx, c, 2, 6)


@pytest.mark.parametrize("L", [10, 20])
def test_scales_that_are_no_powers_of_two_for_many_rows(ctx, L):
    attend(ctx, Caches(L, 4, 256, 128, 64, 64, [75, 21, 40, 33], 16, powers=False), L, 11, prior=True)
    attend(ctx, Caches(L, 4, 256, 128, 64, 64, [200, 9, 0, 129], 32), L, 12, spread=20.0)


def test_keys_that_are_not_numbers_among_many_rows(ctx):
    for L in (10, 20):
        c = Caches(13, 4, 256, 128, 32, 32, [90] * 4, 32)
        c.k.view(torch.uint8)[2, 77, 5, 3] = 0x7f
        q, o, lse = rnd(gen(1), 4 * L, 256 * 32), torch.zeros(4 * L, 256 * 32, device="cuda", dtype=torch.bfloat16), torch.zeros(4, 256, L, device="cuda")
        ctx.ecospa_quant_cache_attn(c.cache, q, o, lse=lse)
        nan = torch.zeros(4, 256, dtype=torch.bool, device="cuda")
        nan[2, 154:156] = True
        assert torch.equal(lse.isnan(), nan[:, :, None].expand(4, 256, L))
        assert torch.equal(o.view(4, L, 256, 32).isnan(), nan[:, None, :, None].expand(4, L, 256, 32))


def test_a_bound_below_the_lengths(ctx):
    attend(ctx, Caches(5, 3, 4, 4, 32, 32, [50, 90, 20], 32, cap=100, own_max=60), 1, 7)
    attend(ctx, Caches(5, 2, 4, 4, 32, 32, [-4, 3], 32, cap=100), 5, 7, prior=True)
    attend(ctx, Caches(5, 2, 4, 4, 32, 32, [0, 0], 32, cap=100, own_max=0), 2, 7, prior=True)


def test_scores_far_apart(ctx):
    attend(ctx, Caches(8, 2, 2, 2, 64, 64, [1500, 900], 64), 1, 8, spread=20.0)


def test_queries_and_keys_that_are_not_numbers(ctx):
    for n, L in ((40, 1), (700, 1), (90, 20)):
        c = Caches(9, 2, 2, 2, 32, 32, [n, n], 32)
        q, o, lse = rnd(gen(1), 2 * L, 64), torch.zeros(2 * L, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(2, 2, L, device="cuda")
        c.k.view(torch.uint8)[0, 1, 5, 3] = 0x7f                         # one key of request 0, head 1
        q[L:, :32] = float("nan")                                       # request 1, head 0
        ctx.ecospa_quant_cache_attn(c.cache, q, o, lse=lse)
        nan = torch.zeros(2, 2, dtype=torch.bool, device="cuda")
        nan[0, 1] = nan[1, 0] = True
        assert torch.equal(lse.isnan(), nan[:, :, None].expand(2, 2, L))
        assert torch.equal(o.view(2, L, 2, 32).isnan(), nan[:, None, :, None].expand(2, L, 2, 32))


def test_the_results_of_other_keys_may_be_the_outputs(ctx):
    c = Caches(11, 2, 4, 2, 64, 96, [500, 3], 64)
    for L in (1, 4):
        q, o_in, lse_in = rnd(gen(2), 2 * L, 4 * 64), rnd(gen(3), 2 * L, 4 * 96), torch.randn(2, 4, L, device="cuda", generator=gen(4))
        o, lse = torch.zeros_like(o_in), torch.zeros_like(lse_in)
        ctx.ecospa_quant_cache_attn(c.cache, q, o, lse=lse, o_in=o_in, lse_in=lse_in)
        ctx.ecospa_quant_cache_attn(c.cache, q, o_in, lse=lse_in, o_in=o_in, lse_in=lse_in)
        assert torch.equal(o, o_in) and torch.equal(lse, lse_in)


# ---- append ------------------------------------------------------------------------------------------------------------------------------
def tables(h_kv, n, e, seed):
    a = torch.rand(h_kv, n, e // 2, device="cuda", generator=gen(seed)) * 6.28
    return a.cos().contiguous(), a.sin().contiguous()


def put(ctx, c, L, seed, rope=True, mul=1.0, change=None, pos=None, tab=400):
    """Appends L random rows and compares everything with the oracle, keys as a cache of bf16 gets them."""
    g = gen(seed)
    qkv = rnd(g, c.B * L, (c.h + c.h_kv) * c.e + c.h_kv * c.f + 8, mul=mul) * torch.exp(torch.randn(c.B * L, 1, device="cuda", generator=g)).bfloat16()
    if change is not None:
        change(qkv)
    pos = (torch.arange(c.B, device="cuda", dtype=torch.int32) * 7 if pos is None else pos) if rope else None
    tabs = tables(c.h_kv, tab, c.e, seed + 1) if rope else None
    q = torch.full((c.B * L, c.h * c.e), 9.0, device="cuda", dtype=torch.bfloat16)
    plain_q = q.clone()
    before, scales_before = c.host(), (c.k_scale.clone(), c.v_scale.clone())
    # the same rows into a cache of bf16: the keys and queries as the library turns them
    pk, pv = (torch.zeros(c.B, c.h_kv, c.cap, d, device="cuda", dtype=torch.bfloat16) for d in (c.e, c.f))
    ctx.ecospa_cache_append(B.KvCache(pk, pv, c.lens, c.h, 1.0), qkv, pos, rope=tabs, q=plain_q)
    ctx.ecospa_quant_cache_append(c.cache, qkv, pos, rope=tabs, q=q)
    assert torch.equal(q.view(torch.int16), plain_q.view(torch.int16))
    keys = host(pk)
    h = lambda t: None if t is None else t.cpu().numpy().astype(np.float64)

    want = {n: x.copy() for n, x in before.items()}
    rows = host(qkv)
    for b in range(c.B):
        first = int(c.lens[b]) - L
        slots = [first + t for t in range(L) if 0 <= first + t < c.cap and (not rope or 0 <= int(pos[b]) + t < tab)]
        for name, src in (("k", keys[b]), ("v", None)):
            for gq in range(c.h_kv):
                for i in sorted({s // c.block for s in slots}):
                    at = [s for s in slots if s // c.block == i]
                    x = np.stack([src[gq, s] if src is not None else rows[b * L + s - first, (c.h + c.h_kv) * c.e + gq * c.f:(c.h + c.h_kv) * c.e + (gq + 1) * c.f] for s in at])
                    codes, scales = want[name][b, gq], want[name + "_scale"][b, gq]
                    s, lo = Q.block_scale(x), max(first, 0)
                    if lo > i * c.block:
                        s = max(s, scales[i])
                        if s > scales[i]:
                            codes[i * c.block:lo] = Q.e4m3(codes[i * c.block:lo] * (scales[i] / s))
                    codes[at] = Q.e4m3(x / s)
                    scales[i] = s
    got = c.host()
    for n in want:
        assert np.array_equal(got[n], want[n], equal_nan=True), (n, np.argwhere(~((got[n] == want[n]) | (np.isnan(got[n]) & np.isnan(want[n]))))[:4])


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("L", [1, 3, 16, 33, 150])
def test_append(ctx, L, block):
    lens = [L, L + 1, L + 15, L + 16, L + 31, L + 32, L + 63, L + 100, L + 127, L + 128]
    put(ctx, Caches(L + block, len(lens), 4, 2, 32, 48, lens, block), L, 20)


@pytest.mark.parametrize("e,f", [(16, 16), (48, 112), (64, 48), (128, 128), (112, 32)])
@pytest.mark.parametrize("rope", [False, True])
def test_append_widths(ctx, e, f, rope):
    put(ctx, Caches(e + f, 3, 6, 3, e, f, [90, 33, 60], 32, layout="tokens"), 30, 21, rope=rope)
    put(ctx, Caches(e + f, 3, 6, 3, e, f, [90, 1, 64], 64), 1, 22, rope=rope)


def test_append_of_tokens_without_a_place(ctx):
    c = Caches(30, 5, 4, 2, 32, 32, [3, 60, 70, 44, 0], 32, cap=64)      # rows before the cache, behind it, none
    put(ctx, c, 10, 23)
    c = Caches(30, 3, 4, 2, 32, 32, [40, 41, 42], 32, cap=64)            # positions outside the tables
    put(ctx, c, 10, 24, pos=torch.tensor([-5, 95, 300], dtype=torch.int32, device="cuda"), tab=100)


def test_scales_rise_and_stay(ctx):
    c = Caches(31, 2, 2, 1, 32, 32, [40, 40], 64, cap=100)
    for i, mul in enumerate((1.0, 1e-3, 300.0, 1e5, 1.0)):               # earlier rows are brought along, down to the type's smallest values
        c.lens += 1
        put(ctx, c, 1, 40 + i, mul=mul)


def test_append_of_extreme_numbers(ctx):
    def change(x):
        x[0] = 0.0
        x[1, ::3] = float("inf")
        x[2, ::5] = float("nan")
        x[3] = 3.3e38
        x[4] = 1e-38
        x[5] = float("nan")
        x[6] = 448.0
        x[7] = 450.0
    for L, lens in ((1, [1] * 8), (8, [20])):
        put(ctx, Caches(33, len(lens), 2, 1, 32, 32, lens, 16, cap=40), L, 25, rope=False, change=change)


def test_appending_token_by_token_and_at_once(ctx):
    """Codes differ by the scales they were first brought to, never by more than a rounding each: the same where sizes do not grow."""
    at_once, one = (Caches(34, 1, 2, 1, 32, 32, [0], 32, cap=64) for _ in range(2))
    qkv = rnd(gen(5), 40, 4 * 32)
    qkv[0] = 8.0                                                          # the largest comes first ...
    qkv[32] = 8.0                                                         # ... in both blocks
    qkv = qkv.clamp(-8, 8)
    at_once.lens += 40
    ctx.ecospa_quant_cache_append(at_once.cache, qkv)
    for t in range(40):
        one.lens += 1
        ctx.ecospa_quant_cache_append(one.cache, qkv[t:t + 1])
    assert torch.equal(at_once.k.view(torch.uint8), one.k.view(torch.uint8)) and torch.equal(at_once.v.view(torch.uint8), one.v.view(torch.uint8))
    assert torch.equal(at_once.k_scale[..., :2], one.k_scale[..., :2])


def test_caches_on_another_stream_and_in_a_graph(ctx):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        other = B.Context("cuda:0", stream)
        c = Caches(35, 3, 4, 2, 64, 64, [600, 300, 20], 64, cap=700)
        qkv, o = rnd(gen(6), 3, 8 * 64), torch.zeros(3, 256, device="cuda", dtype=torch.bfloat16)

        def step():
            c.lens.add_(1)
            other.ecospa_quant_cache_append(c.cache, qkv)
            other.ecospa_quant_cache_attn(c.cache, qkv[:, :256], o)

        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for seed in (7, 8, 9):
            qkv.copy_(rnd(gen(seed), 3, 8 * 64))
            state = [t.clone() for t in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale, c.lens)]
            step()
            want, after = o.clone(), c.k.view(torch.uint8).clone()
            for t, s in zip((c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale, c.lens), state):
                t.copy_(s)
            o.zero_()
            graph.replay()
            stream.synchronize()
            assert torch.equal(o, want) and torch.equal(c.k.view(torch.uint8), after)


@pytest.mark.parametrize("what", ["requests", "rows"])
def test_offsets_beyond_32_bits(ctx, what):
    """Caches whose second request, or whose rows, lie more than 4 GB apart: as the same caches side by side."""
    Bn, h_kv, cap, e, L = 2, 2, 160, 64, 3
    far = (1 << 32) + (1 << 20)
    strides = (far, cap * e, e, 1) if what == "requests" else (e * h_kv, e, (1 << 25) - 64, 1)
    size = sum((n - 1) * s for n, s in zip((Bn, h_kv, cap, e), strides)) + 1
    assert size > 1 << 32
    lens = torch.tensor([cap, cap - 31], dtype=torch.int32, device="cuda")
    qkv = rnd(gen(1), Bn * (cap - 40), (4 + 2 * h_kv) * e)
    more = rnd(gen(2), Bn * L, (4 + 2 * h_kv) * e)
    got = []
    for spread in (False, True):
        k, v = ((torch.empty(size, dtype=torch.uint8, device="cuda").as_strided((Bn, h_kv, cap, e), strides) if spread else
                 torch.empty((Bn, h_kv, cap, e), dtype=torch.uint8, device="cuda")) for _ in range(2))
        k.fill_(0x7f), v.fill_(0x7f)
        ks, vs = (torch.zeros((Bn, h_kv, cap // 16), device="cuda") for _ in range(2))
        now = lens - L
        ctx.ecospa_quant_cache_append(B.QuantCache(k.view(F8), v.view(F8), ks, vs, now, 4, 0.125, 16), qkv)
        cache = B.QuantCache(k.view(F8), v.view(F8), ks, vs, lens, 4, 0.125, 16)
        ctx.ecospa_quant_cache_append(cache, more)
        k[0, :, :40], v[0, :, :40], k[1, :, :9], v[1, :, :9] = 0, 0, 0, 0      # rows in front of what was appended
        ks.masked_fill_(ks == 0, 1.0), vs.masked_fill_(vs == 0, 1.0)
        o, lse = torch.zeros(Bn * L, 4 * e, device="cuda", dtype=torch.bfloat16), torch.zeros(Bn, 4, L, device="cuda")
        ctx.ecospa_quant_cache_attn(cache, more[:, :4 * e], o, lse=lse)
        got.append((k.clone(), v.clone(), ks, vs, o, lse))
        assert torch.isfinite(lse).all()
    for a, b in zip(*got):
        assert torch.equal(a, b)
