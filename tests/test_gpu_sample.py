"""Drawing tokens on the GPU against the fp64 oracle.  Weights are whole numbers of 2^-42 of the best one's binade, each off by half of that and by the
library's exponential, 2^-44 of it: a token or border can differ from the oracle's only where the random number or a bound falls within (V + 2) 2^-41 of
the best one's weight of another answer; there it has to be one of the answers for a random number and bounds moved by as much.  Probabilities: the
same, and half a step of fp32."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2511_11641_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def check(ctx, x, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """x [B, V] on the GPU; parameters: lists or None."""
    Bn, V = x.shape
    f = lambda p, t=torch.float32: None if p is None else torch.tensor(p, dtype=t, device="cuda")
    token, prob = torch.full((Bn,), -9, dtype=torch.int32, device="cuda"), torch.full((Bn,), -9.0, device="cuda")
    ut = f(u)
    args = dict(temperature=f(temperature), top_k=f(top_k, torch.int32), top_p=f(top_p), min_p=f(min_p))
    got = ctx.ecospa_sample(x, ut, token=token, prob=prob, **args)
    assert got is token
    rows = x.float().cpu().numpy()
    host = lambda t, other: [other] * Bn if t is None else t.cpu().double().tolist()
    ps = list(zip(host(ut, 0), host(args["temperature"], 1.0), host(args["top_k"], 0), host(args["top_p"], 1.0), host(args["min_p"], 0.0)))
    tok, pr = token.tolist(), prob.tolist()
    for b, (uu, t, k, p, m) in enumerate(ps):
        p, m, room = 1.0 if np.isnan(p) else p, 0.0 if np.isnan(m) else m, (V + 2) * 2.0 ** -41
        answers = [Q.sample(rows[b], uu, t, int(k), p, m)]
        if answers[0][2] <= room:
            move = [-room, 0.0, room]
            answers += [Q.sample(rows[b], max(uu, 0.0) + du, t, int(k), p + dp if p < 1 else p, m + dm if m > 0 else m)
                        for du in move for dp in (move if p < 1 else [0.0]) for dm in (move if m > 0 else [0.0])]
        assert any(tok[b] == want and abs(pr[b] - share) <= share * 2.0 ** -24 + 2 * room for want, share, _ in answers), (b, tok[b], pr[b], answers, uu, t, k, p, m)
    return token, prob


def rows(seed, Bn, V, dtype=torch.float32, spread=2.5, pitch=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (spread * torch.randn(Bn, pitch or (V + 63) // 64 * 64, device="cuda", generator=g)).to(dtype)
    return x[:, :V], np.random.RandomState(seed)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 511, 512, 513, 1000, 2047, 2048, 2049, 8191, 8193, 32000, 50257])
def test_sizes(ctx, V, dtype):
    x, r = rows(V, 13, V, dtype)
    u = r.rand(13).tolist()
    t = (0.3 + r.rand(13)).tolist()
    check(ctx, x, u)
    check(ctx, x, u, t)
    check(ctx, x, u, t, top_k=r.randint(1, V + 2, 13).tolist())
    check(ctx, x, u, t, top_p=r.rand(13).tolist())
    check(ctx, x, u, t, min_p=(0.2 * r.rand(13)).tolist())
    check(ctx, x, u, t, top_k=r.randint(1, min(V, 60) + 1, 13).tolist(), top_p=(0.5 + 0.5 * r.rand(13)).tolist(), min_p=(0.1 * r.rand(13)).tolist())


@pytest.mark.parametrize("Bn,V", [(300, 20000), (40, 131072), (3, 1 << 20), (1, 262144), (700, 100)])
@pytest.mark.parametrize("spread", [0.5, 4.0])
def test_many_rows_and_large_vocabularies(ctx, Bn, V, spread):
    x, r = rows(Bn, Bn, V, torch.float32 if spread < 1 else torch.bfloat16, spread)
    u = r.rand(Bn).tolist()
    check(ctx, x, u, top_p=(1.0 - 0.3 * r.rand(Bn) ** 2).tolist(), min_p=(0.01 * r.rand(Bn)).tolist())
    check(ctx, x, u, (0.5 + r.rand(Bn)).tolist(), top_k=r.randint(1, V, Bn).tolist(), top_p=(0.6 + 0.4 * r.rand(Bn)).tolist())


@pytest.mark.parametrize("V", [5, 600, 9000, 50000])
def test_equal_logits(ctx, V):
    """Ties at every border go to the lower index; more of them than the list holds."""
    x = torch.full((12, (V + 7) // 8 * 8), 1.5, device="cuda")[:, :V]
    u = [0.0, 0.1, 0.25, 0.5, 0.75, 0.9, 0.99, 0.999999, 0.3, 0.6, 0.7, 0.2]
    check(ctx, x, u)
    check(ctx, x, u, top_k=[1, 2, 3, V // 2 + 1, V, V + 1, 4, 5, V // 3 + 1, V - 1 or 1, 2, 0])
    check(ctx, x, u, top_p=[0.5, 0.25, 0.125, 1.0, 0.75, 0.0, 0.5, 0.5, 0.25, 0.5, 0.75, 0.5], min_p=[1.0] * 12)
    y = torch.full((12, (V + 7) // 8 * 8), 1.5, device="cuda")[:, :V]
    y[:, ::3] = 1.0                      # two values: thousands of ties on either side
    check(ctx, y, u, top_k=[1, V // 2 + 1, V * 2 // 3, V * 2 // 3 + 1, V, 3, 4, 5, V // 3 + 1, 2, V - 1 or 1, 0])
    # sums of two weights fall on no border by accident here
    check(ctx, y, u, top_p=[0.51, 0.27, 0.13, 0.97, 0.73, 0.0, 0.55, 0.59, 0.22, 0.53, 0.77, 0.57])


@pytest.mark.parametrize("n", [100, 200, 255, 256, 300])
def test_top_k_about_what_a_list_of_all_kept_tokens_holds(ctx, n):
    """n tokens in the border's bin, a sixteenth of a binade wide, and as many just below it, which may be taken for its own at first."""
    x = torch.full((8, 3000), -20.0, device="cuda")
    r = np.random.RandomState(n)
    for b in range(8):
        at = r.permutation(3000)
        x[b, at[0]] = 0.0
        x[b, at[1:n + 1]] = -65.0 / 92.332
        x[b, at[n + 1:2 * n + 1]] = -67.8 / 92.332
    k = [1, 2, n // 2, n, n + 1, n + 2, 2 * n, 2 * n + 1]
    u = r.rand(8).tolist()
    check(ctx, x, u, top_k=k)
    check(ctx, x, u, top_k=k, top_p=[0.999, 0.3, 0.7, 0.51, 0.93, 0.77, 0.61, 0.123])
    check(ctx, x, u, top_k=k, min_p=[0.5] * 4 + [0.49] * 4)


def test_one_logit_far_above(ctx):
    x, r = rows(5, 8, 5000)
    x[:, 1234] = 80.0
    check(ctx, x, r.rand(8).tolist(), top_k=[1, 2, 50, 4000, 0, 5, 6, 7], top_p=[1.0, 0.9, 0.5, 1.0, 0.999, 1.0, 0.1, 0.99])
    x[:, 4321] = 80.0                    # two of them in different ranges
    check(ctx, x, r.rand(8).tolist(), top_k=[1, 2, 50, 4000, 0, 5, 6, 7], top_p=[1.0, 0.9, 0.5, 1.0, 0.999, 1.0, 0.1, 0.99])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks_infinities_and_nan(ctx, dtype):
    x, r = rows(6, 9, 9000, dtype)
    inf, nan = float("inf"), float("nan")
    x[0] = -inf
    x[1] = nan
    x[2, :] = -inf
    x[2, 8999] = -3.0                    # one token left
    x[3, ::2] = -inf
    x[4, 5::7] = nan
    x[5, [17, 8500]] = inf
    x[6, 3000:] = -inf                   # whole ranges masked
    x[7, :8192] = -inf
    x[8] = -inf
    x[8, 100] = nan
    u = r.rand(9).tolist()
    for kw in ({}, dict(top_k=[5] * 9), dict(top_p=[0.9] * 9), dict(min_p=[0.05] * 9), dict(top_k=[20] * 9, top_p=[0.8] * 9, min_p=[0.01] * 9), dict(temperature=[0.0] * 9)):
        token, prob = check(ctx, x, u, **kw)
        assert token[[0, 1, 8]].tolist() == [-1] * 3 and prob[[0, 1, 8]].tolist() == [0.0] * 3
        assert int(token[2]) == 8999 and float(prob[2]) == 1.0 and int(token[5]) in (17, 8500)


def test_parameters_at_their_ends(ctx):
    x, r = rows(7, 16, 3000)
    inf, nan = float("inf"), float("nan")
    u = [0.0, -1.0, nan, 1.0, 2.0, inf, -inf, 0.99999994] + r.rand(8).tolist()
    check(ctx, x, u)
    check(ctx, x, u, temperature=[0.0, -1.0, nan, inf, 1e-3, 1e-30, 1e-45, 1e30, 100.0, 0.01, 1.0, -inf, -0.0, 3e38, 1e-10, 2.0])
    check(ctx, x, u, top_p=[0.0, -1.0, nan, 1.0, 2.0, inf, -inf, 1e-30, 0.99999994, 0.5, 0.1, 0.2, 0.3, 1e-8, 0.9, 0.7])
    check(ctx, x, u, min_p=[0.0, -1.0, nan, 1.0, 2.0, inf, -inf, 1e-30, 0.99999994, 0.5, 0.1, 0.2, 0.3, 1e-8, 0.9, 0.7])
    check(ctx, x, u, top_k=[0, -1, 1, 2, 3000, 3001, 2999, 2 ** 31 - 1, -2 ** 31, 5, 6, 7, 8, 9, 10, 11])
    x.mul_(1e30)
    check(ctx, x, u)
    x.mul_(1e-38).mul_(1e-22)
    check(ctx, x, u, top_p=[0.5 + 0.03 * i for i in range(16)])


def test_the_best_token_is_the_processed_logits_pick(ctx):
    x, _ = rows(8, 50, 32000, torch.bfloat16)
    pick, _ = ctx.ecospa_logits_process(x)
    token = ctx.ecospa_sample(x, torch.rand(50, device="cuda"), temperature=torch.zeros(50, device="cuda"))
    assert torch.equal(pick, token)
    assert torch.equal(pick, ctx.ecospa_sample(x, torch.rand(50, device="cuda"), top_k=torch.ones(50, dtype=torch.int32, device="cuda")))


def test_shares_of_the_tokens(ctx):
    """Evenly spaced random numbers give every token its share, to one draw."""
    V, n = 37, 4096
    x, _ = rows(9, 1, V)
    u = (torch.arange(n, device="cuda").float() + 0.5) / n
    token, prob = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    many = torch.zeros(n, 64, device="cuda")
    many[:, :V] = x
    ctx.ecospa_sample(many[:, :V], u, token=token, prob=prob)
    share = torch.softmax(x[0].double(), 0)
    got = torch.bincount(token.long(), minlength=V)
    assert bool((got - n * share).abs().max() <= 1.0001) and bool((token[1:] >= token[:-1]).all())
    assert torch.allclose(prob.double(), share[token.long()], rtol=2.0 ** -23)


def test_on_another_stream_and_in_a_graph(ctx):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        other = B.Context("cuda:0", stream)
        x, _ = rows(10, 20, 40000)
        u, token = torch.rand(20, device="cuda"), torch.zeros(20, dtype=torch.int32, device="cuda")
        p = torch.full((20,), 0.9, device="cuda")
        k = torch.full((20,), 300, device="cuda", dtype=torch.int32)
        step = lambda: other.ecospa_sample(x, u, top_k=k, top_p=p, token=token)
        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for seed in (11, 12, 13):
            x.copy_(rows(seed, 20, 40000)[0])
            u.copy_(torch.rand(20, device="cuda"))
            step()
            want = token.clone()
            token.zero_()
            graph.replay()
            stream.synchronize()
            assert torch.equal(token, want)


@pytest.mark.parametrize("V,dtype", [(300, torch.float32), (3000, torch.bfloat16), (20000, torch.float32), (70000, torch.bfloat16)])
def test_restrictions_together_with_temperatures_at_their_ends(ctx, V, dtype):
    x, r = rows(V + 1, 16, V, dtype)
    x[3, V // 3] = float("inf")
    x[4, [5, V // 2, V - 1]] = float("inf")
    x[5, ::2] = -float("inf")
    x[6, : V - 40] = -float("inf")
    x[7] *= 1e-3
    x[8] *= 30.0
    t = [1e-3, 1e-30, 1e30, 1.0, 0.5, 100.0, 1e-6, 1.0, 1.0, 0.02, 3e38, 1e-45, 5.0, 0.2, 2.0, 0.7]
    for seed in range(6):
        r = np.random.RandomState(seed + V)
        k = [int(v) for v in np.exp(r.rand(16) * np.log(V)).astype(int)]
        check(ctx, x, r.rand(16).tolist(), t, top_k=k, top_p=(1.0 - 0.6 * r.rand(16) ** 2).tolist(), min_p=(0.2 * r.rand(16) ** 3).tolist())
        check(ctx, x, r.rand(16).tolist(), t, top_k=k, min_p=(10.0 ** (-8 * r.rand(16))).tolist())
        check(ctx, x, r.rand(16).tolist(), t, top_p=r.rand(16).tolist(), min_p=(10.0 ** (-8 * r.rand(16))).tolist())
