"""Every kernel of the attention over a shared prefix, in every way a call is cut for it, against the fp64 oracle: outputs, log-sum-exp and weights of
all requests.  Five requests differ, the others repeat them (results may differ by roundings: rows of a wavefront move their reference together).
Bounds: see test_gpu_serving.py."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2511_11641_amd import binding as B
from prefix_attn_kinds import CASES, chosen, lengths
from test_gpu_serving import Case, ctx  # noqa: F401 (ctx: the fixture)
from util import host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel,form,shape", CASES, ids=["-".join(map(str, k + f)) + "-" + "_".join(map(str, s)) for k, f, s in CASES])
def test_every_kernel(ctx, kernel, form, shape):  # noqa: F811
    Bn, L, h, h_kv, e, f, P, own_max = shape
    few = min(Bn, 5)
    c = Case(sum(shape), few, L, h, h_kv, e, f, P, lengths(few, L, own_max), cap=own_max + 3)
    want = S.prefix_attn(host(c.q), host(c.k), host(c.v), c.lens.tolist(), h, c.scale, host(c.pk), host(c.pv), host(c.w))
    of = torch.arange(Bn, device="cuda") % few
    k, v, w, lens = (x[of].contiguous() for x in (c.k, c.v, c.w, c.lens))
    cache = B.KvCache(k, v, lens, h, c.scale, c.pk, c.pv, own_max=own_max)
    assert chosen(B.load(), cache.desc, L) == (kernel, form)
    q = c.q.view(few, L * h * e)[of].view(Bn * L, h * e)
    o = torch.full((Bn * L, h * f), float("nan"), device="cuda", dtype=torch.bfloat16)
    lse, w_out = torch.full((Bn, h, L), float("nan"), device="cuda"), torch.full_like(w, -7.0)
    ctx.ecospa_prefix_attn(cache, q, o, lse=lse, weights=w, weights_out=w_out)
    of = of.cpu().numpy()
    empty = np.isinf(want["lse"])
    d = 2.0 ** -17 * want["s_abs"] + 2.0 ** -21 * (1 + np.where(empty, 0, np.abs(want["lse"])))
    moved = np.repeat(np.expm1(2 * d).transpose(0, 2, 1).reshape(few * L, h), f, axis=1)
    room = 2.0 ** -8 * np.abs(want["o"]) + (2.0 ** -8 + 2.0 ** -12 + moved) * want["av"]
    rows = lambda x: x.reshape(few, L, h * f)[of].reshape(Bn * L, h * f)
    assert (np.abs(host(o) - rows(want["o"])) <= rows(room)).all()
    got = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(got), empty[of])
    sees = ~empty[of]
    assert (np.abs(got[sees] - want["lse"][of][sees]) <= d[of][sees]).all()
    got, alive = w_out.double().cpu().numpy(), np.broadcast_to(np.arange(c.cap) < lens.cpu().numpy()[:, None, None], w.shape)
    room = (want["w"] - host(c.w)) * np.expm1(4 * d.max()) + 2.0 ** -20 * (want["w"] + 1e-3)
    assert (got[~alive] == -7.0).all() and (np.abs(got - want["w"][of])[alive] <= room[of][alive]).all()


@pytest.mark.parametrize("e,f", [(16, 32), (48, 32), (64, 64), (80, 16), (128, 128)])
@pytest.mark.parametrize("L,h,h_kv,P,lens", [(131, 8, 2, 67, [131, 200, 40, 0, 333]), (520, 4, 4, 0, [520, 530]), (33, 16, 1, 129, [33, 70, 5])])
def test_weights_of_many_rows(ctx, e, f, L, h, h_kv, P, lens):  # noqa: F811
    """512 rows of a request and more: the weights by 64 keys a workgroup, from keys and queries read again."""
    c = Case(e + L, len(lens), L, h, h_kv, e, f, P, lens)
    assert L * h // h_kv >= 512
    c.check(*c.run(ctx))
