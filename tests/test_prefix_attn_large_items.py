"""Which prompts go on items of 256 rows (csrc/prefix_attn.hip): those whose rows fill them as well as items of 128, with keys enough (host only)."""
import pytest

from paper_2511_11641_amd import binding as B
from test_prefix_attn_cuts import cut

LARGE, SMALL = 4, 3


@pytest.mark.parametrize("kind,shape", [
    (LARGE, (16, 509, 32, 8, 64, 64, 8192, 509)), (LARGE, (20, 500, 32, 8, 64, 64, 2000, 500)), (LARGE, (64, 128, 32, 8, 32, 64, 4096, 178)),
    (LARGE, (64, 128, 32, 8, 64, 32, 1000, 178)), (LARGE, (96, 128, 32, 8, 32, 32, 8192, 178)),
    # 384 rows of a request in place of 512, 128 in place of 256: as much less work
    (SMALL, (64, 300, 16, 16, 32, 32, 2000, 400)), (SMALL, (64, 300, 16, 16, 32, 32, 8192, 400)), (SMALL, (128, 128, 8, 8, 48, 64, 3000, 300)),
    (SMALL, (130, 65, 16, 4, 64, 64, 4096, 70)),
    # few keys
    (SMALL, (64, 250, 16, 16, 64, 32, 500, 250)), (SMALL, (64, 512, 16, 16, 32, 32, 0, 512)), (SMALL, (192, 256, 16, 16, 32, 32, 1000, 306)),
    # less than two rounds of workgroups, wide heads
    (SMALL, (10, 509, 32, 8, 64, 64, 8192, 509)), (SMALL, (64, 128, 32, 8, 64, 128, 4096, 178))])
def test_items_of_256_rows(kind, shape):
    a, _ = cut(B.load(), *shape)
    assert a["slots"] == 0 and a["own"] == kind
