"""What the server and its command refuse before they touch a GPU."""
import pytest
import torch

from paper_2511_11641_amd import serve


@pytest.mark.parametrize("more", [[], ["--cache-block", "64", "--quant-weights"]])
def test_a_temperature_without_a_draw(more, capsys):
    with pytest.raises(SystemExit) as e:
        serve.main(["--temperature", "0.7", *more])
    assert e.value.code == 2 and "--top-p" in capsys.readouterr().err


@pytest.mark.parametrize("only", ["u", "temperature", "top_k", "top_p", "min_p"])
def test_draws_by_numbers_in_host_memory(only):
    """A kernel would read what isn't there."""
    there = lambda t: type("OnGpu", (), {"shape": t.shape, "dtype": t.dtype, "is_cuda": True, "contiguous": lambda self: self})()
    args = {"u": torch.zeros(4, 2), "temperature": torch.ones(2), "top_k": torch.ones(2, dtype=torch.int32), "top_p": torch.ones(2), "min_p": torch.zeros(2)}
    args = {n: t if n == only else there(t) for n, t in args.items()}
    srv = object.__new__(serve.Server)
    srv._room = lambda L: None
    with pytest.raises(ValueError, match="on the GPU"):
        srv.generate(torch.zeros((2, 3), dtype=torch.long), 4, **args)
