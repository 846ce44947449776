"""Products in 8-bit integers and rows brought to 8 bits whose operands and results lie behind the first 4 GB."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2511_11641_amd import binding as B

pytestmark = pytest.mark.gpu
BORDER = 1 << 32


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def _near(got, want, slack):
    return (np.abs(got.float().cpu().numpy() - want) <= np.abs(want) * 2.0 ** -8 + slack * 2.0 ** -24 * (1 + 2.0 ** -8) + 1e-38).all()


@pytest.mark.parametrize("M", [3, 64, 300])
def test_weights_beyond_4_gb(ctx, M):
    N, K = 66000, 65536
    w = torch.empty((N, K), dtype=torch.int8, device="cuda")
    w.view(torch.int32).copy_(torch.arange(N * K // 4, device="cuda", dtype=torch.int32).view(N, K // 4).mul_(-1640531527))
    sw = torch.rand(N, device="cuda", generator=torch.Generator(device="cuda").manual_seed(M)) * 1e-3
    a = torch.randint(-127, 128, (M, K), device="cuda", dtype=torch.int8, generator=torch.Generator(device="cuda").manual_seed(M))
    sa = torch.full((M,), 0.01, device="cuda")
    y = ctx.ecospa_contract_quant(a, sa, w, sw)
    assert 65516 * K < BORDER < 65556 * K and (N - 40) * K > BORDER
    for first in (65516, N - 40):      # rows on both sides of the border, and the last ones
        part = slice(first, first + 40)
        want, slack = Q.contract_quant(a.cpu().numpy()[-3:], sa.cpu().numpy()[-3:], w[part].cpu().numpy(), sw[part].cpu().numpy())
        assert _near(y[-3:, part], want, slack)


@pytest.mark.parametrize("N,K,act", [(136, 256, B.ACT_NONE), (1040, 512, B.ACT_SWIGLU), (24832, 2048, B.ACT_NONE), (24832, 2048, B.ACT_GELU_ERF), (24832, 2048, B.ACT_SWIGLU)])
def test_rows_and_results_beyond_4_gb(ctx, N, K, act):
    """Rows far apart in both: as the same rows side by side, and nothing written between them."""
    M, lda, ldc = 300, (1 << 24) - 16, (1 << 23) - 8
    g = torch.Generator(device="cuda").manual_seed(N)
    packed = torch.randint(-127, 128, (M, K), device="cuda", dtype=torch.int8, generator=g)
    w = torch.randint(-127, 128, (N, K), device="cuda", dtype=torch.int8, generator=g)
    sa, sw, bias = (torch.rand(n, device="cuda", generator=g) * 0.01 for n in (M, N, N))
    bias = bias.bfloat16()
    width = N // 2 if act == B.ACT_SWIGLU else N
    a = torch.zeros(M * lda, dtype=torch.int8, device="cuda").view(M, lda)[:, :K]
    a.copy_(packed)
    whole = torch.full((M, ldc), 3.0, dtype=torch.bfloat16, device="cuda")
    assert (M - 45) * lda < BORDER < (M - 40) * lda and 2 * 256 * ldc < BORDER < 2 * 257 * ldc
    ctx.ecospa_contract_quant(a, sa, w, sw, bias=bias, act=act, out=whole[:, :width])
    want = ctx.ecospa_contract_quant(packed, sa, w, sw, bias=bias, act=act)
    assert torch.equal(whole[:, :width], want)
    assert bool((whole[:, width:] == 3.0).all())
    rows = [0, 255, 256, 257, 299]
    exact, slack = Q.contract_quant(packed.cpu().numpy()[rows], sa.cpu().numpy()[rows], w[:80].cpu().numpy(), sw[:80].cpu().numpy(), bias[:80].float().cpu().numpy(), act)
    assert _near(want[rows][:, :exact.shape[1]], exact, slack)


def test_codes_beyond_4_gb(ctx):
    rows, cols = 70000, 65536
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    for first in (0, 65530, rows - 6):
        x[first:first + 12] = torch.randn(x[first:first + 12].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(first)).bfloat16()
    assert 65535 * cols < BORDER <= 65536 * cols
    q, s = ctx.ecospa_quant_rows(x)
    for first in (0, 65530, rows - 6):
        wq, ws = Q.quant_rows(x[first:first + 12].float().cpu().numpy())
        assert np.array_equal(q[first:first + 12].cpu().numpy(), wq) and np.array_equal(s[first:first + 12].cpu().numpy(), ws)
    assert not bool(s[12:65530].any()) and not bool(q[12:65530].any())
