"""The serving harness at its limits: positions end with the tables, with or without evictions, and what is refused changes nothing."""
import pytest
import torch

from paper_2511_11641_amd import binding as B
from paper_2511_11641_amd.serve import Server
from test_gpu_serve import VOCAB, _stack

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def ids(*shape, seed=1):
    return torch.randint(0, VOCAB, shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("gated", [True, False])
def test_positions_end_with_the_tables(ctx, gated):
    srv = Server(_stack(ctx, gated, 32, d_h=64), 2, 16, 32)
    with pytest.raises(AssertionError, match="position"):
        srv.set_prefix(ids(33))
    srv.set_prefix(ids(20))
    srv.feed(ids(2, 9))
    srv.evict(4, 2)                                      # positions go on counting: 29 of 32 are used
    with pytest.raises(AssertionError, match="position"):
        srv.feed(ids(2, 4))
    assert srv.lens.tolist() == [4, 4] and srv.pos.tolist() == [29, 29]
    assert torch.isfinite(srv.feed(ids(2, 3))).all()     # the last position there is
    with pytest.raises(AssertionError, match="position"):
        srv.feed(ids(2, 1))
    assert srv.lens.tolist() == [7, 7] and srv.pos.tolist() == [32, 32]
    srv.set_prefix(ids(32))                              # all of them the prefix's
    with pytest.raises(AssertionError, match="position"):
        srv.feed(ids(2, 1))


def test_generating_past_the_tables(ctx):
    srv = Server(_stack(ctx, True, 8), 2, 8, 24)
    srv.set_prefix(ids(10))
    with pytest.raises(AssertionError, match="position"):
        srv.generate(ids(2, 5), 11, keep=4, recent=1)    # the last token is not fed: 10 + 5 + 10 positions
    assert srv.lens.tolist() == [0, 0] and srv.pos.tolist() == [10, 10]
    assert srv.generate(ids(2, 5), 10, keep=4, recent=1).shape == (2, 10) and srv.pos.tolist() == [24, 24]


def test_tokens_of_another_batch(ctx):
    srv = Server(_stack(ctx, True, 8), 3, 8, 24)
    srv.set_prefix(ids(10))
    with pytest.raises(AssertionError, match="requests"):
        srv.feed(ids(2, 5))
    assert srv.lens.tolist() == [0, 0, 0] and srv.pos.tolist() == [10, 10, 10]
