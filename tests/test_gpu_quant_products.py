"""Rows of 8-bit integers and their products against the fp64 oracle, through every kernel that a product can run on."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2511_11641_amd import binding as B
from util import GemmDesc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def _rows(rows, cols, seed, dtype=torch.bfloat16, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols + pad, generator=g) * torch.exp(0.5 * torch.randn(1, cols + pad, generator=g))
    return x.to(dtype)


def _check_rows(ctx, x, want_pad=0):
    rows, cols = x.shape
    pitch = (cols + 15) // 16 * 16 + want_pad
    q = torch.full((rows + 1, pitch), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows + 1,), 7.0, device="cuda")
    ctx.ecospa_quant_rows(x.cuda() if not x.is_cuda else x, q[:rows, :cols], s[:rows])
    wq, ws = Q.quant_rows(x.float().cpu().numpy())
    assert np.array_equal(s[:rows].cpu().numpy(), ws, equal_nan=True)
    assert np.array_equal(q[:rows, :cols].cpu().numpy(), wq)
    assert float(s[rows]) == 7.0 and bool((q[rows] == 77).all()) and bool((q[:rows, cols:] == 77).all())      # nothing beside the rows


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 8), (1, 512), (3, 24), (5, 2048), (7, 2056), (2, 4104), (9, 16392), (3, 40000), (1025, 1000), (1100, 1032), (1030, 2040), (1027, 4096),
                                       (1029, 4104)])
def test_rows(ctx, rows, cols, dtype):
    _check_rows(ctx, _rows(rows, cols, rows + cols, dtype), want_pad=16)


def test_rows_of_a_wider_matrix(ctx):
    x = _rows(6, 200, 1, pad=56).cuda()
    _check_rows(ctx, x[:, 56:])


def test_rows_at_the_borders_of_numbers(ctx):
    x = _rows(13, 64, 2, torch.float32)
    x[0] = 0.0
    x[1, 5] = float("inf")
    x[2, 63] = float("nan")
    x[3] *= 1e-30
    x[4] *= 1e-37
    x[5] = 0.0
    x[5, 7] = 1e-45            # a subnormal maximum: 1e-45 / 127 is zero
    x[6] *= 1e37
    x[7, 9] = -3.4e38
    x[8] = torch.arange(64) - 31.5          # quotients half-way between codes
    x[8, 0] = 127.0
    x[9] = -0.0
    x[10] = 2.0 ** -149 * torch.arange(64)
    x[11, 0] = float("-inf")
    x[12] = 2.0 ** -149 * 3 * torch.arange(64)          # a maximum of 189 steps: a scale of one
    _check_rows(ctx, x)


# sizes and the kernel they run on: each tile shape of the ring (0 .. 11), the resident workgroups (12), and K shared out (13 .. 16)
SIZES = [
    (4611, 2592, 192, 0), (1751, 4832, 192, 1), (4039, 2824, 192, 2), (1156, 4888, 192, 3), (4665, 1544, 192, 4), (1433, 5400, 192, 5),
    (964, 5464, 192, 6), (4798, 784, 192, 7), (391, 4656, 192, 8), (269, 5456, 192, 9), (134, 5552, 224, 10), (73, 5024, 192, 11),
    (9, 8, 1808, 13), (1, 4824, 192, 14), (2, 80, 288, 15), (35, 4192, 224, 16), (1, 1024, 512, 15), (3, 16, 16, 15),
    (3129, 3896, 16, 0), (61, 3088, 2048, 14), (64, 5504, 2048, 16), (33, 32000, 256, 9), (129, 136, 64, 15), (8144, 5504, 2048, 12),
    (6150, 6152, 4096, 12), (2049, 2056, 8208, 7)]


def _route(ctx, M, N, K, act):
    g = GemmDesc(B.BF16, M, N, K // 2, 1 << 32, K // 2, 0, 2 << 32, K // 2, 0, 0, 1, None)
    g.epi.kind = {B.ACT_NONE: 0, B.ACT_SWIGLU: 6}.get(act, 4)
    g.epi.act, g.epi.c, g.epi.ldc, g.epi.c2, g.epi.ldc2 = act, 3 << 32, N, 3 << 32, N
    return ctx.lib._Z17ecospa_gemm_routeRK8GemmDesc(C.byref(g))


def _check_product(ctx, M, N, K, act, bias, seed, rows_checked=400):
    g = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.randint(-127, 128, (M, K), device="cuda", generator=g, dtype=torch.int8)
    b = torch.randint(-127, 128, (N, K + 16), device="cuda", generator=g, dtype=torch.int8)[:, 16:]
    sa = torch.rand(M, device="cuda", generator=g) * 0.02 + 1e-4
    sb = (torch.rand(N, device="cuda", generator=g) * 0.02 + 1e-4) / 16
    bv = torch.randn(N, device="cuda", generator=g).bfloat16() if bias else None
    width = N // 2 if act == B.ACT_SWIGLU else N
    out = torch.full((M + 2, width + 8), 5.0, device="cuda", dtype=torch.bfloat16)
    got = ctx.ecospa_contract_quant(a, sa, b, sb, bias=bv, act=act, out=out[1:M + 1, :width])
    rows = np.unique(np.linspace(0, M - 1, min(M, rows_checked)).astype(int))
    h = lambda t: t.cpu().numpy()
    # the products of the checked rows, exact in 64 bits
    want, slack = Q.contract_quant(h(a)[rows], h(sa)[rows], h(b), h(sb), None if bv is None else h(bv.float()), act)
    y = h(got.float())[rows].astype(np.float64)
    bad = np.abs(y - want) - (np.abs(want) * 2.0 ** -8 + slack * 2.0 ** -24 * (1 + 2.0 ** -8) + 1e-38)
    assert bad.max() <= 0, (bad.max(), np.unravel_index(bad.argmax(), bad.shape))
    assert bool((out[0] == 5.0).all()) and bool((out[-1] == 5.0).all()) and bool((out[:, width:] == 5.0).all())


@pytest.mark.parametrize("M,N,K,route", SIZES)
def test_products(ctx, M, N, K, route):
    assert _route(ctx, M, N, K, B.ACT_NONE) == route
    _check_product(ctx, M, N, K, B.ACT_NONE, True, M)
    _check_product(ctx, M, N, K, B.ACT_NONE, False, M + 1, 60)


@pytest.mark.parametrize("act", [B.ACT_GELU_ERF, B.ACT_GELU_TANH, B.ACT_SWIGLU])
@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (5, 2048, 1024), (61, 5504, 2048), (333, 1040, 336), (1000, 2000, 512), (4100, 2048, 2752), (6145, 6160, 2048)])
def test_activations(ctx, M, N, K, act):
    _check_product(ctx, M, N, K, act, M % 2 == 1, M + act, 40)


def test_every_kernel_is_among_them(ctx):
    tried = {_route(ctx, M, N, K, B.ACT_NONE) for M, N, K, _ in SIZES}
    assert tried == set(range(17))


def test_sums_at_their_largest(ctx):
    a = torch.full((5, 131056), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(8, device="cuda")
    y = ctx.ecospa_contract_quant(a, one[:5], a[:1].expand(8, -1).contiguous(), one)
    assert bool((y == torch.tensor(float(131056 * 16384)).bfloat16().cuda()).all())      # below 2^31: no sum has turned over


def test_rows_that_are_not_numbers_say_so(ctx):
    x = _rows(4, 64, 5).cuda()
    x[2, 3] = float("nan")
    q, s = ctx.ecospa_quant_rows(x)
    w, sw = ctx.ecospa_quant_rows(_rows(32, 64, 6).cuda())
    y = ctx.ecospa_contract_quant(q, s, w, sw)
    assert bool(y[2].isnan().all()) and bool(y[[0, 1, 3]].isfinite().all())


def test_on_another_stream_and_in_a_graph(ctx):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        other = B.Context("cuda:0", stream)
        x, w = _rows(70, 512, 7).cuda(), _rows(96, 512, 8).cuda()
        wq, sw = other.ecospa_quant_rows(w)
        q, s, y = torch.zeros(70, 512, dtype=torch.int8, device="cuda"), torch.zeros(70, device="cuda"), torch.zeros(70, 96, dtype=torch.bfloat16, device="cuda")

        def step():
            other.ecospa_quant_rows(x, q, s)
            other.ecospa_contract_quant(q, s, wq, sw, out=y)

        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for seed in (9, 10, 11):
            x.copy_(_rows(70, 512, seed))
            step()
            want = y.clone()
            y.zero_()
            graph.replay()
            stream.synchronize()
            assert torch.equal(y, want)


def test_codes_of_a_row_out_of_a_wider_matrix(ctx):
    """A single row counts as dense whatever its stride; the codes made for it have a pitch of their own."""
    x = _rows(4, 608, 7).cuda()
    for part in (x[1:2, 8:520], x[1:2, :600], x[:, 8:520]):
        q, s = ctx.ecospa_quant_rows(part)
        wq, ws = Q.quant_rows(part.float().cpu().numpy())
        assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws) and q.stride(0) % 16 == 0


@pytest.mark.parametrize("M", [3, 300])
def test_operands_and_results_beyond_4_gb(ctx, M):
    """Rows of weights and of activations brought to 8 bits that lie behind the first 4 GB."""
    N, K = 66000, 65536
    w = torch.empty((N, K), dtype=torch.int8, device="cuda")
    w.view(torch.int32).copy_(torch.arange(N * K // 4, device="cuda", dtype=torch.int32).view(N, K // 4).mul_(-1640531527))
    sw, last = torch.rand(N, device="cuda") * 1e-3, N - 520
    a, sa = ctx.ecospa_quant_rows(_rows(M, K, M).cuda())
    y = ctx.ecospa_contract_quant(a, sa, w, sw)
    want, slack = Q.contract_quant(a.cpu().numpy()[:4], sa.cpu().numpy()[:4], w[last:last + 40].cpu().numpy(), sw[last:last + 40].cpu().numpy())
    got = y[:4, last:last + 40].float().cpu().numpy()
    assert (np.abs(got - want) <= np.abs(want) * 2.0 ** -8 + slack * 2.0 ** -24 * (1 + 2.0 ** -8) + 1e-38).all()
    del w, y
    x = torch.zeros((40000, 65536), dtype=torch.bfloat16, device="cuda")
    x[39990:] = _rows(10, 65536, 9).cuda()
    q, s = ctx.ecospa_quant_rows(x)
    wq, ws = Q.quant_rows(x[39990:].float().cpu().numpy())
    assert np.array_equal(q[39990:].cpu().numpy(), wq) and np.array_equal(s[39990:].cpu().numpy(), ws) and not bool(s[:39990].any())
