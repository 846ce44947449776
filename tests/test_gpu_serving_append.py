"""New tokens into the caches without a query output (the queries are read from the projection's own rows): every element of both caches and of the
accumulated weights, from zeroed ones, against the oracle - written rows, rows that stay as they were, tokens without a row."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2511_11641_amd import binding as B
from test_gpu_serving import ctx, gen, rnd  # noqa: F401 (ctx: the fixture)
from util import host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("Bn,L,h,h_kv,e,f,cap,lens", [
    (1, 1, 1, 1, 16, 16, 1, [1]), (4, 1, 16, 16, 32, 32, 40, [1, 40, 7, 0]), (3, 5, 8, 2, 48, 128, 20, [5, 20, 3]), (2, 70, 6, 3, 128, 64, 90, [70, 95]),
    (5, 1, 4, 4, 16, 80, 9, [9, 10, -1, 3, 1]), (1, 600, 24, 8, 64, 64, 600, [600]), (2, 3, 12, 1, 80, 16, 4, [4, 2])])
def test_append_without_a_query_output(ctx, Bn, L, h, h_kv, e, f, cap, lens, layout):  # noqa: F811
    g = gen(Bn * L + cap)
    qkv = rnd(g, Bn * L, (h + h_kv) * e + h_kv * f + 16)[:, :-16]
    assert (qkv != 0).all()                              # a zero in a cache is a row that was not written
    shape = lambda n: (Bn, h_kv, cap, n) if layout == "heads" else (Bn, cap, h_kv, n)
    new = lambda n: torch.zeros(shape(n), device="cuda", dtype=torch.bfloat16) if layout == "heads" else torch.zeros(shape(n), device="cuda", dtype=torch.bfloat16).transpose(1, 2)
    k, v, w = new(e), new(f), torch.rand(Bn, h_kv, cap, device="cuda", generator=g) + 0.5
    want = S.append(host(qkv), host(k), host(v), lens, h, w=host(w))
    cache = B.KvCache(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"), h, 0.1)
    rows = qkv.clone()
    ctx.ecospa_cache_append(cache, qkv, weights=w)
    written = [sum(0 <= n - L + t < cap for t in range(L)) for n in lens]
    assert np.count_nonzero(want[1]) == sum(written) * h_kv * e and np.count_nonzero(want[2]) == sum(written) * h_kv * f
    assert np.array_equal(host(k), want[1]) and np.array_equal(host(v), want[2]) and np.array_equal(host(w), want[3])
    assert torch.equal(qkv, rows), "the rows of the projection are read only"
