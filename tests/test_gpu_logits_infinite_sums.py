"""log sum exp of rows with infinities: infinite where all is a number, not a number where something is not - in one workgroup's range, or in several."""
import pytest
import torch

from paper_2511_11641_amd import binding as B

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


@pytest.mark.parametrize("V", [9, 1000, 9000, 30000, 200000])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_infinities_beside_what_is_not_a_number(ctx, V, dt):
    first, last = 1, V - 1
    x = torch.zeros(8, (V + 7) // 8 * 8, device="cuda", dtype=dt)[:, :V]
    x[0, last] = INF
    x[1, first], x[1, last] = INF, INF
    x[2, first], x[2, last] = INF, NAN
    x[3, first], x[3, last] = NAN, INF
    x[4], x[4, last] = -INF, INF
    x[5], x[5, last] = -INF, NAN
    x[6, first], x[6, last] = -INF, INF
    x[7, last], x[7, last - 1] = INF, NAN
    pick, lse = ctx.ecospa_logits_process(x)
    want = torch.logsumexp(x.double(), 1).float()
    assert torch.isnan(want).tolist() == [False, False, True, True, False, True, False, True]
    assert torch.equal(torch.isnan(lse), torch.isnan(want)) and torch.equal(lse[~torch.isnan(want)], want[~torch.isnan(want)])
    assert pick.tolist() == [last, first, first, last, last, -1, last, last]
