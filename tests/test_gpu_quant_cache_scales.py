"""Attention over caches of 8-bit floats whose scales are any positive numbers, down to the smallest."""
import pytest
import torch

from paper_2511_11641_amd import binding as B
from test_gpu_quant_cache import Caches, attend, gen, rnd

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


LENS = [1, 15, 33, 50, 77, 200]
KINDS = [(3, 3, 32, 32, 1), (8, 2, 64, 64, 3), (4, 1, 96, 128, 20), (2, 2, 128, 48, 70)]      # heads, widths, new tokens


@pytest.mark.parametrize("size", [2.0 ** -149, 1e-42, 3e-39, 2.0 ** -126, 1e-30])
@pytest.mark.parametrize("h,h_kv,e,f,L", KINDS)
def test_keys_of_tiny_scales(ctx, h, h_kv, e, f, L, size):
    """Scores next to zero: every key that a query sees weighs the same, and those it doesn't see nothing."""
    c = Caches(1, len(LENS), h, h_kv, e, f, LENS, 16)
    c.k_scale.mul_(0.0).add_(size)
    attend(ctx, c, L, 2, prior=L == 3)
    attend(ctx, c, L, 3, spread=1e30)


@pytest.mark.parametrize("size", [2.0 ** -127, 1.3 * 2.0 ** -127, 1.9 * 2.0 ** -126, 1.5 * 2.0 ** -118, 1.7 * 2.0 ** -101, 1.1 * 2.0 ** -99, 1.7 * 2.0 ** 100])
@pytest.mark.parametrize("h,h_kv,e,f,L", KINDS)
def test_values_of_scales_at_the_ends(ctx, h, h_kv, e, f, L, size):
    """Codes of 256 and more, so that what comes out is above bf16's least normal number."""
    c = Caches(4, len(LENS), h, h_kv, e, f, LENS, 32)
    c.v_scale.mul_(0.0).add_(size)
    codes = (256 + 192 * torch.rand(c.v.shape, device="cuda", generator=gen(5))).to(F8).view(torch.uint8)
    live = torch.arange(c.cap, device="cuda") < torch.tensor(LENS, device="cuda")[:, None]
    c.v.view(torch.uint8).copy_(torch.where(live[:, None, :, None], codes, 0x7f))
    attend(ctx, c, L, 6)


def test_keys_of_large_scales(ctx):
    c = Caches(7, len(LENS), 4, 2, 64, 64, LENS, 64, powers=False)
    c.k_scale.mul_(2.0 ** 100)
    attend(ctx, c, 2, 8, spread=2.0 ** -100)


def test_scales_of_zero_make_rows_of_zero(ctx):
    """What a cache of zeros holds where no token was put."""
    c = Caches(9, 2, 2, 2, 32, 32, [40, 70], 16)
    c.k.view(torch.uint8)[:, :, :16] = 0
    c.v.view(torch.uint8)[:, :, :16] = 0
    c.k_scale[:, :, 0] = 0.0
    c.v_scale[:, :, 0] = 0.0
    attend(ctx, c, 5, 10)
    c.lens.fill_(9)
    o, lse = torch.ones(4, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(2, 2, 2, device="cuda")
    ctx.ecospa_quant_cache_attn(c.cache, rnd(gen(1), 4, 64), o, lse=lse)
    assert not bool(o.any()) and torch.allclose(lse, torch.tensor([8.0, 9.0], device="cuda").log(), rtol=2.0 ** -21)
