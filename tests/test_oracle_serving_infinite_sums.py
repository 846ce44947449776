"""The oracle's log sum exp of rows with infinities against the definition (CPU)."""
import numpy as np
import torch

from oracle import serving_oracle as S

INF, NAN = np.inf, np.nan


def test_sums_with_infinities_and_what_is_not_a_number():
    x = np.array([[0, INF, 1], [INF, INF, 0], [INF, NAN, 0], [NAN, 1, INF], [-INF, NAN, -INF], [-INF, 2, -INF], [-INF, -INF, -INF], [NAN, NAN, NAN], [1, 2, NAN]])
    with np.errstate(all="ignore"):
        _, pick, lse = S.logits_process(x)
    assert np.array_equal(lse, torch.logsumexp(torch.from_numpy(x), 1).numpy(), equal_nan=True)
    assert pick.tolist() == [1, 0, 0, 2, -1, 1, -1, -1, 1]
