"""Appends to caches of 8-bit floats behind rows that others brought to 8 bits, at scales that are no powers of two, and appends against the oracle's own."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2511_11641_amd import binding as B
from test_gpu_quant_cache import Caches, gen, put, rnd
from util import host

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


@pytest.mark.parametrize("block", [16, 128])
@pytest.mark.parametrize("mul", [1e-3, 1.0, 300.0, 1e5])
def test_behind_rows_of_any_scales(ctx, block, mul):
    put(ctx, Caches(block, 6, 4, 2, 48, 64, [9, 20, 31, 90, 120, 3], block, powers=False), 3, 20, mul=mul)
    put(ctx, Caches(block, 3, 4, 2, 128, 128, [100, 131, 90], block, powers=False), 60, 21, mul=mul)


def _one_block(scale, values, d=16):
    """A block that holds one earlier row, of `values`, at this scale; the second row is to come."""
    k, v = (torch.zeros(1, 1, 16, d, dtype=torch.uint8, device="cuda") for _ in range(2))
    for t in (k, v):
        t[0, 0, 0] = torch.tensor(values, device="cuda").to(F8).view(torch.uint8)
    ks, vs = (torch.tensor([[[scale]]], dtype=torch.float32, device="cuda") for _ in range(2))
    lens = torch.tensor([2], dtype=torch.int32, device="cuda")
    return B.QuantCache(k.view(F8), v.view(F8), ks, vs, lens, 1, 1.0, 16)


def test_quotients_half_way_between_codes(ctx):
    """Numbers that are odd multiples of half a step times a scale, which is no power of two and a last place off: to the nearest code, as if by an exact division."""
    for m in range(129, 256, 2):
        for step in (-1, 0, 1):
            s = np.float32(m / 128.0)
            s = s if step == 0 else np.nextafter(s, np.float32(9.0 if step > 0 else 0.0))
            x = np.array([m / 128.0 * 2.0 ** e for e in (-10, -9, -8, -7)] + [m / 128.0 * n * 2.0 ** -10 for n in (3, 5, 7, 9)] + [m / 128.0 * n / 16.0 for n in (17, 19, 21, 23, 25, 27, 29, 31)])
            x = torch.from_numpy(x).bfloat16()
            c = _one_block(float(s), [0.0] * 16)
            qkv = torch.cat((torch.zeros(16), x.float(), x.float())).bfloat16().cuda()[None]
            ctx.ecospa_quant_cache_append(c, qkv)
            assert float(c.k_scale) == float(s)
            want = Q.e4m3(x.double().numpy() / np.float64(s))
            assert np.array_equal(host(c.k[0, 0, 1]), want) and np.array_equal(host(c.v[0, 0, 1]), want), (m, step)


def test_earlier_rows_next_to_half_way_between_codes(ctx):
    """Codes times a scale that come within fp32's rounding of half a step, on either side of it, when the block's scale rises."""
    codes = [8.0 + i for i in range(8)] + [-(8.0 + i) for i in range(8)]
    tried = 0
    for c in range(9, 16, 2):
        for t in range(17, 32, 2):
            for off in (-7, -5, -3, -2, -1, 1, 2, 3, 5, 7):      # fp32's last place of c s is 8 or 16 of these
                whole = next((t * (1 << j) + off for j in range(18, 26) if (t * (1 << j) + off) % c == 0 and 1 << 23 <= (t * (1 << j) + off) // c < 1 << 24), None)
                if whole is None:
                    continue
                s = np.float32(whole // c) * np.float32(2.0 ** -23)      # c s is within one part in 2^24 of t 2^n
                cache = _one_block(float(s), codes)
                qkv = torch.full((1, 48), 7000.0, device="cuda").bfloat16()
                ctx.ecospa_quant_cache_append(cache, qkv)
                after = np.float64(float(cache.k_scale))
                assert after == 16.0
                want = Q.e4m3(np.array(codes) * (np.float64(s) / after))
                assert np.array_equal(host(cache.k[0, 0, 0]), want) and np.array_equal(host(cache.v[0, 0, 0]), want), (c, t, off)
                tried += 1
    assert tried >= 20


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("L", [1, 3, 40])
def test_appends_are_the_oracles(ctx, L, rope, block):
    """Everything that an append leaves, against the oracle's own append: quarter turns keep keys and queries exact."""
    lens = [L, L + 1, L + 15, L + 31, L + 90, L - 1, 70]
    c = Caches(L + block, len(lens), 6, 2, 48, 32, lens, block, cap=128)
    g = gen(L)
    qkv = rnd(g, c.B * L, (c.h + c.h_kv) * c.e + c.h_kv * c.f) * torch.exp(torch.randn(c.B * L, 1, device="cuda", generator=g)).bfloat16()
    pos, tabs = None, None
    if rope:
        pos = torch.tensor([0, 5, -2, 130, 90, 7, 0], dtype=torch.int32, device="cuda")
        turn = torch.randint(0, 4, (c.h_kv, 140, c.e // 2), device="cuda", generator=g)
        tabs = tuple(torch.tensor(x, device="cuda")[turn].contiguous() for x in ([1.0, 0.0, -1.0, 0.0], [0.0, 1.0, 0.0, -1.0]))
    h = lambda t: None if t is None else t.cpu().numpy().astype(np.float64)
    want_q, want = Q.append(host(qkv), c.host(), lens, c.h, block, None if pos is None else pos.tolist(), *(h(t) for t in tabs or (None, None)))
    q = torch.full((c.B * L, c.h * c.e), 9.0, device="cuda", dtype=torch.bfloat16)
    ctx.ecospa_quant_cache_append(c.cache, qkv, pos, rope=tabs, q=q)
    got = c.host()
    for n in want:
        assert np.array_equal(got[n], want[n], equal_nan=True), n
    assert np.array_equal(host(q), want_q)
