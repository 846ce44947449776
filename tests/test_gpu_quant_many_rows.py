"""Rows brought to 8 bits, more of them than one launch takes."""
import pytest
import torch

from paper_2511_11641_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [(1 << 23) + 1, (1 << 25) + 3, (1 << 26) + 5])
def test_rows_by_the_ten_million(ctx, rows, dtype):
    """2^26 rows of a wavefront each are 2^32 work-items."""
    x = torch.randn((rows, 8), dtype=dtype, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    q, s = torch.full((rows + 1, 16), 77, dtype=torch.int8, device="cuda"), torch.full((rows + 1,), 7.0, device="cuda")
    ctx.ecospa_quant_rows(x, q[:rows, :8], s[:rows])
    for part in torch.arange(0, rows, 1 << 24).tolist():
        at = slice(part, min(part + (1 << 24), rows))
        top = x[at].abs().amax(1).float()
        want = top / torch.full_like(top, 127.0)      # (by a number, torch multiplies with its reciprocal)
        assert torch.equal(s[at], want)
        assert torch.equal(q[at, :8].float(), torch.round(x[at].float() / want[:, None].masked_fill(want[:, None] == 0, 1.0)))
    assert bool((q[:, 8:] == 77).all()) and bool((q[rows] == 77).all()) and float(s[rows]) == 7.0
