"""What the server's command refuses before it touches a GPU."""
import pytest

from paper_2511_11641_amd import serve


@pytest.mark.parametrize("more", [[], ["--cache-block", "64", "--quant-weights"]])
def test_a_temperature_without_a_draw(more, capsys):
    with pytest.raises(SystemExit) as e:
        serve.main(["--temperature", "0.7", *more])
    assert e.value.code == 2 and "--top-p" in capsys.readouterr().err
