"""Requests that share no prefix: a harness that was just built takes their tokens."""
import numpy as np
import pytest
import torch

from paper_2511_11641_amd import binding as B
from paper_2511_11641_amd.serve import Server
from test_gpu_serve import VOCAB, _stack
from util import host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [True, False])
def test_a_new_harness_without_a_prefix(gated):
    st = _stack(B.Context("cuda:0"), gated, 20, d_h=64)
    ids = torch.randint(0, VOCAB, (2, 20), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    want = [host(st.forward(ids[b].contiguous())) for b in range(2)]
    srv = Server(st, 2, 24, 20)
    for at, n in ((0, 18), (18, 1), (19, 1)):
        got = host(srv.feed(ids[:, at:at + n].contiguous()))
        for b in range(2):
            assert np.linalg.norm(got[b] - want[b][at + n - 1]) / np.linalg.norm(want[b][at + n - 1]) < 2e-2, (b, at)
    assert srv.pos.tolist() == [20, 20]
    srv = Server(st, 2, 24, 40 if gated else 20)
    assert srv.generate(ids[:, :5], 8).shape == (2, 8)
