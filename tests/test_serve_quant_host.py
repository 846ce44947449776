"""What the serving harness refuses before it touches a GPU: caches in 8 bits that should be evictable, and draws without their random numbers."""
import pytest
import torch

from paper_2511_11641_amd.serve import Server


def test_caches_in_8_bits_keep_no_weights_to_evict_by():
    with pytest.raises(ValueError, match="evictable"):
        Server(None, 1, 16, 16, cache_block=16)


@pytest.mark.parametrize("only", ["top_k", "top_p", "min_p"])
def test_restrictions_need_random_numbers(only):
    with pytest.raises(ValueError, match="random numbers"):
        Server.generate(object.__new__(Server), torch.zeros((2, 3), dtype=torch.long), 4, **{only: torch.ones(2)})


@pytest.mark.parametrize("u", [torch.zeros(4), torch.zeros(2, 4), torch.zeros(4, 2, dtype=torch.float64)], ids=lambda t: f"{tuple(t.shape)}-{t.dtype}")
def test_random_numbers_of_another_shape(u):
    srv = object.__new__(Server)
    srv._room = lambda L: None
    with pytest.raises(ValueError, match="random numbers"):
        srv.generate(torch.zeros((2, 3), dtype=torch.long), 4, u=u)
