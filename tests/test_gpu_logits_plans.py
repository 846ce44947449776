"""Logits of every type into every type where rows are many: vocabularies of several workgroups a row, and one workgroup of 32 logits a thread.  Values
that fp32 holds exactly at every step: results are equal, the best token too."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2511_11641_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


@pytest.mark.parametrize("Bn,V", [(43, 50257), (163, 20001), (129, 16385), (257, 32768), (2, 131072)])
@pytest.mark.parametrize("dt,odt", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_every_plan(ctx, Bn, V, dt, odt):
    distinct, H = min(Bn, 4), 700
    rng = np.random.default_rng(V)
    of = np.arange(Bn) % distinct
    x = rng.integers(-64, 65, (distinct, V)) / 8.0
    x[1, [V - 1, V - 7]] = 40.0                          # the lower of equal ones, at the end
    hist = rng.integers(-1, V + 1, (distinct, H))
    hist[1] %= V - 7
    hist[:, ::3] = hist[:, :1]
    ids = rng.integers(0, V - 7, (distinct, 20))
    ids[:, 7] = ids[:, 2]
    mask = rng.integers(0, 1 << 32, (2, (V + 31) // 32), dtype=np.uint64).astype(np.uint32).view(np.int32)
    ref = dict(history=hist, history_len=np.array([H, 600, 1, 0])[:distinct], repetition=np.array([1, 2, 4, 2])[:distinct],
               frequency=np.array([0.25, 0, 0.5, 1])[:distinct], presence=np.array([0.5, 0, 0.25, 1])[:distinct],
               temperature=np.array([1, 2, 0.5, 4])[:distinct], bias_ids=ids, bias=rng.integers(-8, 9, (distinct, 20)) / 4.0, mask=mask,
               mask_row=np.array([0, -1, 1, 2])[:distinct])
    want, pick, lse = S.logits_process(x, **ref)
    whole = ("history", "history_len", "bias_ids", "mask", "mask_row")
    up = lambda n, a: torch.from_numpy(np.ascontiguousarray(a if n == "mask" else a[of])).to(torch.int32 if n in whole else torch.float32).cuda()
    pitch = (V + 7) // 8 * 8 + 8
    buf = torch.full((Bn, pitch), float("nan"), device="cuda", dtype=TYPES[dt])
    buf[:, :V] = torch.from_numpy(x[of]).to(TYPES[dt]).cuda()
    out = torch.full((Bn, pitch), 77.0, device="cuda", dtype=TYPES[odt])
    got_pick, got_lse = ctx.ecospa_logits_process(buf[:, :V], out=out[:, :V], **{n: up(n, a) for n, a in ref.items()})
    assert torch.equal(out[:, :V].cpu(), torch.from_numpy(want[of]).float().to(TYPES[odt])) and (out[:, V:] == 77).all()
    assert got_pick.tolist() == pick[of].tolist() and pick[1] == V - 7
    assert (np.abs(got_lse.double().cpu().numpy() - lse[of]) <= 2.0 ** -19 * (2 + np.abs(lse[of]))).all()
