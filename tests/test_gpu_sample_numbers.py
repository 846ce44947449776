"""Random numbers and shares of a draw with all the bits that fp32 gives them, down to the smallest: equal logits of 0 weigh 2^42 units each, so every sum, bound and draw is a
whole number worked out in fractions."""
from fractions import Fraction
from math import ceil, floor

import pytest
import torch

from paper_2511_11641_amd import binding as B
from test_gpu_sample import check

pytestmark = pytest.mark.gpu
UNIT = 1 << 42


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def numbers(n, seed):
    """fp32 in [0, 1) of every exponent, subnormal ones too, with all 24 bits in use."""
    g = torch.Generator().manual_seed(seed)
    bits = torch.randint(0, 0x3f800000, (n,), generator=g)
    bits[::2] = torch.randint(0x28000000, 0x3f800000, ((n + 1) // 2,), generator=g)      # from 2^-47 on, where they decide
    return bits.to(torch.int32).view(torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [2, 200, 5000, 1 << 17, 1 << 20])
@pytest.mark.parametrize("by_k", [False, True])
def test_equal_tokens(ctx, V, dtype, by_k):
    n = 64
    u, p = numbers(n, V), numbers(n, V + 1)
    u[:3] = torch.tensor([2.0 ** -33, 1 - 2.0 ** -24, 2.0 ** -149])
    p[3:40] = (torch.randint(1, V + 1, (37,)).double() / V).float()      # near a border of tokens, as near as fp32 comes from either side
    p[3:12] = torch.nextafter(p[3:12], torch.zeros(9))
    p[12:24] = torch.nextafter(p[12:24], torch.ones(12))
    p[40] = 2.0 ** -20 * (1 + 2.0 ** -23)
    p = p.clamp(max=1 - 2.0 ** -24)
    k = torch.randint(1, V + 1, (n,), dtype=torch.int32) if by_k else torch.full((n,), V, dtype=torch.int32)
    x = torch.zeros((1, (V + 7) // 8 * 8), device="cuda", dtype=dtype).expand(n, -1).contiguous()[:, :V]
    prob = torch.zeros(n, device="cuda")
    token = ctx.ecospa_sample(x, u.cuda(), top_k=k.cuda() if by_k else None, top_p=p.cuda(), prob=prob).tolist()
    alone = ctx.ecospa_sample(x, u.cuda()).tolist()
    for b in range(n):
        ub, pb, kb = Fraction(u[b].item()), Fraction(p[b].item()), int(k[b])
        kept = -(-max(ceil(pb * kb * UNIT), 1) // UNIT)
        assert token[b] == floor(ub * kept * UNIT) // UNIT and prob[b].item() == torch.tensor(1.0 / kept, dtype=torch.float64).float().item(), (b, token[b], u[b], p[b], kb, kept)
        assert alone[b] == floor(ub * V * UNIT) // UNIT, (b, alone[b], u[b])


def test_random_numbers_below_2_to_the_minus_32(ctx):
    """A first token of a share as small as they are: drawn up to it, the next one beyond."""
    x = torch.full((24, 40), -float("inf"), device="cuda")
    small = torch.arange(8, device="cuda") % 8 + 31.0
    x[:, 5] = -0.6931471805599453 * small.repeat(3)
    x[:, 17] = 0.0
    share = torch.sigmoid(x[:, 5].double())
    u = torch.cat((share[:8] * 0.7, share[8:16] * 1.4, share[16:] * 3.1)).float()
    token, _ = check(ctx, x, u.tolist())
    assert token.tolist() == [5] * 8 + [17] * 16
