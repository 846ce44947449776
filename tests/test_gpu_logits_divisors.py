"""Temperatures and repetition penalties that a division can meet - zero, infinite, so small or so large that their reciprocal is not a normal number -
against the quotient and the product in fp64.

Bound: one rounding of the quotient by a product with the rounded reciprocal and a correction, less than 2 units in the last place: 2^-22 of the value,
and two of the smallest steps of fp32 (2^-148) where it is below the normal numbers."""
import numpy as np
import pytest
import torch

from paper_2511_11641_amd import binding as B

pytestmark = pytest.mark.gpu

DIVISORS = [0.0, -0.0, 1e-45, 1e-40, -1e-40, 2.0 ** -128, 2.0 ** -126, 0.7, -1.3, 2.0 ** 126, 3e38, float("inf"), -float("inf")]
VALUES = [0.0, -0.0, 1.0, -1.0, 2.5, -3.25, 1e-3, -7e-5, 1e-30, -1e-38, 1e-42, 1e30, -2e38, 3.4e38, float("inf"), -float("inf"), float("nan")]


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def rows(V):
    return np.resize(np.array(VALUES, dtype=np.float32), (len(DIVISORS), V))


def check(got, ref, what):
    with np.errstate(all="ignore"):
        got, fit = got.double().cpu().numpy(), ref.astype(np.float32).astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(fit)), (what, np.argwhere(np.isnan(got) != np.isnan(fit))[:4])
    inf = np.isinf(fit) | np.isinf(got)
    assert np.array_equal(got[inf], fit[inf]), what
    fine = np.isfinite(fit)
    assert (np.abs(got[fine] - ref[fine]) <= 2.0 ** -22 * np.abs(ref[fine]) + 2.0 ** -148).all(), what


def best(x):
    """(lowest token with the largest value, -1: none; log sum exp) of fp64 rows."""
    ok = np.where(np.isnan(x), -np.inf, x)
    return [int(r.argmax()) if r.max() > -np.inf else -1 for r in ok], torch.logsumexp(torch.from_numpy(x), 1).numpy()


@pytest.mark.parametrize("V", [40, 20000, 200000])
@pytest.mark.parametrize("control", ["temperature", "repetition"])
def test_divisors(ctx, V, control):
    x = rows(V)
    if control == "repetition":
        x[-2:, 1::2] = np.abs(x[-2:, 1::2])
    d = np.array(DIVISORS, dtype=np.float32)
    with np.errstate(all="ignore"):
        quotient, product = x.astype(np.float64) / d[:, None].astype(np.float64), x.astype(np.float64) * d[:, None].astype(np.float64)
    kw = {control: torch.from_numpy(d).cuda()}
    if control == "temperature":
        ref = quotient
    else:
        ref = np.where(x > 0, quotient, product)
        kw["history"] = torch.arange(V, dtype=torch.int32, device="cuda").repeat(len(d), 1)
    logits = torch.from_numpy(x).cuda()
    out = torch.empty_like(logits)
    pick, lse = ctx.ecospa_logits_process(logits, out=out, **kw)
    check(out, ref, control)
    picks, sums = best(out.double().cpu().numpy())      # of the values that came out
    assert pick.tolist() == picks
    got = lse.double().cpu().numpy()
    fine = np.isfinite(sums)
    assert np.array_equal(np.isnan(got), np.isnan(sums)) and np.array_equal(got[np.isinf(sums)], sums[np.isinf(sums)])
    assert (np.abs(got - sums)[fine] <= 2.0 ** -19 * (2 + np.abs(sums[fine]))).all()


def test_a_temperature_of_zero_leaves_a_token(ctx):
    """x / 0 is an infinity of the sign of x: the first positive logit is the pick, and nothing is a number by accident."""
    x = torch.linspace(-3, 2, 1001, device="cuda").flip(0)[:1000].clone().view(1, -1)
    out = torch.empty_like(x)
    pick, lse = ctx.ecospa_logits_process(x, out=out, temperature=torch.zeros(1, device="cuda"))
    assert pick.item() == 0 and lse.item() == float("inf") and torch.equal(out, torch.where(x > 0, float("inf"), -float("inf")))
    pick, lse = ctx.ecospa_logits_process(-x.flip(1).contiguous() - 2.5, temperature=torch.zeros(1, device="cuda"))
    assert pick.item() == int((-x.flip(1) - 2.5 > 0).int().argmax())
