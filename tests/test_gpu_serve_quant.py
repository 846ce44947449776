"""The serving harness with caches and weights in 8 bits and with tokens drawn by given random numbers.

What 8 bits do to logits has no bound worth testing (it depends on how large scores are), so the run is tested link by link: every call of the operators that
a feed makes is compared with the fp64 oracle on the call's own inputs, within the bounds of the operators' own tests, and each call's input has to be what
the call in front of it left.  As a whole: of all the logits of the sequence, those at the position are the nearest."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2511_11641_amd import binding as B
from paper_2511_11641_amd.serve import Server, main
from test_gpu_serve import VOCAB, _stack
from util import host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def ids(*shape, seed=1):
    return torch.randint(0, VOCAB, shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


CONFIGS = [(True, 4, 32, (1, 2)), (True, 2, 64, (3, 4)), (False, 4, 64, (1, 2)), (True, 1, 128, (1, 1))]


@pytest.mark.parametrize("gated,h_kv,d_h,keep", CONFIGS)
@pytest.mark.parametrize("block,weights", [(16, False), (None, True), (64, True)])
@pytest.mark.parametrize("P,prompt", [(0, 37), (70, 5), (200, 1)])
def test_logits_are_nearest_to_those_of_the_position(ctx, gated, h_kv, d_h, keep, block, weights, P, prompt):
    Bsz, steps = 3, 4
    total = P + prompt + steps - 1
    st = _stack(ctx, gated, total, h_kv, d_h, keep)
    x = ids(Bsz, total, seed=P + 1)
    x[:, :P] = x[:1, :P]
    want = [host(st.forward(x[b].contiguous())) for b in range(Bsz)]
    srv = Server(st, Bsz, 48, total, evictable=False, cache_block=block, quant_weights=weights)
    if P:
        srv.set_prefix(x[0, :P].contiguous())
    at = P
    for n in [prompt] + [1] * (steps - 1):
        got = host(srv.feed(x[:, at:at + n].contiguous()))
        at += n
        for b in range(Bsz):
            near = [np.linalg.norm(w - got[b][None], axis=1) for w in want]
            assert (int(np.argmin([n.min() for n in near])), int(near[b].argmin())) == (b, at - 1)
    assert srv.lens.tolist() == [at - P] * Bsz and srv.pos.tolist() == [at] * Bsz


class Tap:
    """The calls of some methods of a context: inputs as they were, and outputs."""

    def __init__(self, ctx, *names):
        self.ctx, self.names, self.calls = ctx, names, []

    def __enter__(self):
        for n in self.names:
            setattr(self.ctx, n, self._tap(n, getattr(self.ctx, n)))
        return self

    def __exit__(self, *_):
        for n in self.names:
            delattr(self.ctx, n)

    def _tap(self, name, f):
        copy = lambda t: t.clone() if isinstance(t, torch.Tensor) else t

        def call(*a, **k):
            before = [copy(t) for t in a], {n: copy(t) for n, t in k.items()}
            r = f(*a, **k)
            self.calls.append((name, *before, tuple(copy(t) for t in r) if isinstance(r, tuple) else copy(r)))
            return r

        return call


def check_rows(x, q, s):
    wq, ws = Q.quant_rows(x.float().cpu().numpy())
    assert np.array_equal(s.flatten().cpu().numpy(), ws) and np.array_equal(q.cpu().numpy(), wq)


def check_product(q, s, w, sw, bias, act, y):
    n = lambda t: None if t is None else t.float().cpu().numpy()
    want, slack = Q.contract_quant(q.cpu().numpy(), n(s.flatten()), w.cpu().numpy(), n(sw), n(bias), B.ACT_NONE if act is None else act)
    assert (np.abs(host(y) - want) <= np.abs(want) * 2.0 ** -8 + slack * 2.0 ** -24 * (1 + 2.0 ** -8) + 1e-38).all()


def check_attention(cache, lens, q, front, lse_front, o):
    c = {"k": cache["k"], "v": cache["v"], "k_scale": cache["ks"], "v_scale": cache["vs"]}
    want = Q.attn(host(q), c, lens, cache["h"], cache["scale"], cache["block"], None if front is None else host(front), None if front is None else lse_front.view(len(lens), cache["h"], -1).double().cpu().numpy())
    L = q.shape[0] // len(lens)
    d = 2.0 ** -17 * want["s_abs"] + 2.0 ** -21 * (1 + np.abs(want["lse"]))
    moved = np.repeat(np.expm1(2 * d).transpose(0, 2, 1).reshape(len(lens) * L, cache["h"]), c["v"].shape[3], axis=1)
    assert (np.abs(host(o) - want["o"]) <= 2.0 ** -8 * np.abs(want["o"]) + (2.0 ** -8 + 2.0 ** -12 + moved) * want["av"]).all()


@pytest.mark.parametrize("gated,h_kv,d_h,keep", CONFIGS)
@pytest.mark.parametrize("P", [0, 70])
def test_every_call_of_a_feed(ctx, gated, h_kv, d_h, keep, P):
    Bsz, n_layers, L = 3, 2, (21, 1)
    st = _stack(ctx, gated, 100, h_kv, d_h, keep)
    srv, x = Server(st, Bsz, 48, 100, evictable=False, cache_block=16, quant_weights=True), ids(Bsz, 22)
    if P:
        srv.set_prefix(ids(P, seed=9))
    done = 0
    names = ("ecospa_quant_rows", "ecospa_contract_quant", "ecospa_quant_cache_append", "ecospa_prefix_attn", "ecospa_quant_cache_attn")
    for n in L:
        with Tap(ctx, *names) as tap:
            logits = srv.feed(x[:, done:done + n].contiguous()).clone()
        done += n
        per = ["rows", "product", "append"] + (["prefix"] if P else []) + ["attn", "rows", "product", "rows", "product", "rows", "product"]
        short = {"ecospa_quant_rows": "rows", "ecospa_contract_quant": "product", "ecospa_quant_cache_append": "append", "ecospa_prefix_attn": "prefix", "ecospa_quant_cache_attn": "attn"}
        assert [short[c[0]] for c in tap.calls] == per * n_layers + ["rows", "product"]
        calls, lens = iter(tap.calls), np.full(Bsz, done)
        for ly in srv.layers + [None]:
            weights = (("wqkv", "bqkv_c", "attn"), ("wo", "bo", "attn"), ("w1", "b1_c", "ffn"), ("w2", "b2", "ffn")) if ly else (("lm", None, None),)
            last = None
            for name, bias, blk in weights:
                _, a, _, (codes, scale) = next(calls)
                if last is not None and name != "w1":
                    assert torch.equal(a[0], last)                  # (a norm stands in front of w1, and of wqkv)
                check_rows(a[0], codes, scale)
                _, (q8, s8, w8, sw), k, y = next(calls)
                mine = ly["quant"][name] if ly else srv.lm_quant
                assert torch.equal(q8, codes) and torch.equal(s8, scale) and torch.equal(w8, mine[0]) and torch.equal(sw, mine[1])
                check_rows({"wqkv": lambda: ly["attn"].wqkv_c, "wo": lambda: ly["attn"].wo_c, "w1": lambda: ly["ffn"].w1_c, "w2": lambda: ly["ffn"].w2_c, "lm": lambda: st.lm.w}[name](), w8, sw)
                own = getattr(ly[blk], bias) if bias else None
                assert (k["bias"] is None) == (own is None) and (own is None or torch.equal(k["bias"], own)) and k["act"] == (ly["ffn"].act if name == "w1" else None)
                check_product(q8, s8, w8, sw, k["bias"], k["act"], y)
                last = y
                if name == "wqkv":
                    _, a, k, _ = next(calls)
                    assert a[0] is ly["cache"] and torch.equal(a[1], last) and a[2].tolist() == [P + done - n] * Bsz
                    front = lse = None
                    if P:
                        _, (shared, _, _, lse_out), _, front = next(calls)
                        assert shared is ly["shared"] and shared.pk is ly["prefix"][0]
                    _, (cache, q, _), k, o = next(calls)
                    assert cache is ly["cache"] and (k["o_in"] is None) == (not P)
                    if P:
                        assert torch.equal(k["o_in"], front)
                    f = lambda t: t.float().cpu().numpy().astype(np.float64)
                    dead = np.arange(48)[None, None, :, None] >= done
                    held = dict(k=np.where(dead, 0, f(ly["kv"][0])), v=np.where(dead, 0, f(ly["kv"][1])), ks=f(ly["scales"][0]), vs=f(ly["scales"][1]), h=cache.h, scale=cache.scale, block=16)
                    if not gated:
                        assert torch.equal(q, last)
                    check_attention(held, lens, q[:, :cache.nq], k["o_in"], k["lse_in"], o)
                    last = o
        assert torch.equal(logits, last)


def test_caches_hold_what_the_oracle_appends(ctx):
    """What a prompt and two single tokens leave in the first layer's caches, from the projections that the library itself made."""
    st = _stack(ctx, False, 64, d_h=64)
    srv, x = Server(st, 2, 40, 64, evictable=False, cache_block=16), ids(2, 25)
    ly = srv.layers[0]
    c = ly["cache"]
    n, lens = c.cap, np.zeros(2, dtype=np.int64)
    want = dict(k=np.zeros((2, c.h_kv, n, c.kq)), v=np.zeros((2, c.h_kv, n, c.kv)))
    rows = [[], []]
    for cut in ((0, 23), (23, 24), (24, 25)):
        kept = {}
        append = ctx.ecospa_quant_cache_append

        def tap(cache, qkv, *a, **k):
            if cache is c:
                kept["qkv"] = qkv.clone()
            return append(cache, qkv, *a, **k)

        ctx.ecospa_quant_cache_append = tap
        try:
            srv.feed(x[:, cut[0]:cut[1]].contiguous())
        finally:
            del ctx.ecospa_quant_cache_append
        for b in range(2):
            rows[b].append(host(kept["qkv"]).reshape(2, -1, kept["qkv"].shape[1])[b])
    for b in range(2):
        r = np.concatenate(rows[b])
        k = r[:, c.h * c.kq:(c.h + c.h_kv) * c.kq].reshape(-1, c.h_kv, c.kq).transpose(1, 0, 2)
        v = r[:, (c.h + c.h_kv) * c.kq:].reshape(-1, c.h_kv, c.kv).transpose(1, 0, 2)
        for name, codes, scales, w in (("k", ly["kv"][0], ly["scales"][0], k), ("v", ly["kv"][1], ly["scales"][1], v)):
            s = scales[b].double().cpu().numpy().repeat(16, axis=1)[:, :25, None]
            got = codes[b, :, :25].float().double().cpu().numpy() * s
            # a code is within 2^-4 of its value, or half of the least code, 2^-10, of the scale; one brought to a later scale is rounded a second time
            assert (np.abs(got - w) <= 2 * np.maximum(np.abs(w) * 2.0 ** -4, s * 2.0 ** -10)).all(), (b, name)
            assert (s <= np.maximum(np.abs(w).reshape(c.h_kv, 25, -1).max() / 224, 2.0 ** -100)).all()      # the least power of two: not above twice of what is needed


@pytest.mark.parametrize("block,weights", [(None, False), (32, True)])
def test_generated_tokens_are_the_draws_of_the_oracle(ctx, block, weights):
    Bsz, steps = 3, 12
    st = _stack(ctx, True, 8)
    srv, prefix, prompts = Server(st, Bsz, 32, 100, evictable=False, cache_block=block, quant_weights=weights), ids(33), ids(Bsz, 6, seed=2)
    f = lambda *v: torch.tensor(v, device="cuda")
    u = torch.rand((steps, Bsz), device="cuda", generator=torch.Generator(device="cuda").manual_seed(7))
    args = dict(u=u, temperature=f(0.7, 1.0, 1.3), top_k=f(0, 20, 200).int(), top_p=f(0.9, 1.0, 0.95), min_p=f(0.0, 0.01, 0.02), repetition=f(1.2, 1.0, 1.5))
    seen, sample = [], ctx.ecospa_sample

    def tap(logits, *a, **k):
        seen.append(logits.clone())
        return sample(logits, *a, **k)

    srv.set_prefix(prefix)
    ctx.ecospa_sample = tap
    try:
        out = srv.generate(prompts, steps, **args)
    finally:
        del ctx.ecospa_sample
    srv.set_prefix(prefix)
    assert torch.equal(out, srv.generate(prompts, steps, **args)), "not the same twice"
    off = 0
    for i in range(steps):
        x = seen[i].cpu().numpy()
        for b in range(Bsz):
            token, _, near = Q.sample(x[b], float(u[i, b]), float(args["temperature"][b]), int(args["top_k"][b]), float(args["top_p"][b]), float(args["min_p"][b]))
            assert out[b, i] == token or near <= (VOCAB + 2) * 2.0 ** -41, (i, b)
    # one token left, or no temperature: the best one, as without a draw
    srv.set_prefix(prefix)
    best = srv.generate(prompts, steps)
    for only in (dict(top_k=torch.ones(Bsz, dtype=torch.int32, device="cuda")), dict(temperature=torch.zeros(Bsz, device="cuda")), dict(min_p=torch.ones(Bsz, device="cuda"))):
        srv.set_prefix(prefix)
        got = srv.generate(prompts, steps, u=u, **only)
        assert torch.equal(best, got), only


def test_masked_tokens_are_never_drawn(ctx):
    srv, prompts = Server(_stack(ctx, True, 8), 3, 32, 64, evictable=False, cache_block=128, quant_weights=True), ids(3, 6)
    words = torch.zeros((2, VOCAB // 32), dtype=torch.int32)
    words[0, 3] = 0x0f0f                                     # row 1: everything masked
    u = torch.rand((10, 3), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    out = srv.generate(prompts, 10, u=u, mask=words.cuda(), mask_row=torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda"))
    assert set(out[0].tolist()) <= {96 + v for v in (0, 1, 2, 3, 8, 9, 10, 11)} and out[1].tolist() == [-1] * 10 and len(set(out[2].tolist())) > 3


def test_full_caches_in_8_bits_are_refused_and_nothing_changes(ctx):
    srv, x = Server(_stack(ctx, True, 8), 2, 8, 64, evictable=False, cache_block=16), ids(2, 9)
    srv.feed(x[:, :7].contiguous())
    with pytest.raises(AssertionError, match="full"):
        srv.feed(x[:, :2].contiguous())
    with pytest.raises(AssertionError, match="without the attention weights"):
        srv.evict(4, 2)
    assert srv.lens.tolist() == [7, 7] and srv.pos.tolist() == [7, 7]
    assert torch.isfinite(srv.feed(x[:, 7:8].contiguous())).all()


def test_a_step_in_a_graph(ctx):
    """The operators of a decoding step, one behind the other as they are used, captured once and replayed: every replay as the eager step."""
    Bsz, h, h_kv, d, kp, V, block = 4, 8, 2, 256, 32, 1000, 16
    nqkv = (h + h_kv) * kp + h_kv * kp
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        own = B.Context("cuda:0")
        weights = [own.ecospa_quant_rows(0.1 * rnd(*s)) for s in ((nqkv, d), (d, h * kp), (V, d))]
        emb = rnd(V, d)
        u = torch.rand((7, Bsz), device="cuda", generator=g)

        def fresh():
            f8 = torch.float8_e4m3fn
            k, v = (torch.zeros((Bsz, h_kv, 64, kp), device="cuda").to(f8) for _ in range(2))
            ks, vs = (torch.zeros((Bsz, h_kv, 4), device="cuda") for _ in range(2))
            lens = torch.tensor([1, 15, 16, 40], dtype=torch.int32, device="cuda")
            return B.QuantCache(k, v, ks, vs, lens, h, kp ** -0.5, block), torch.zeros((Bsz,), dtype=torch.int32, device="cuda"), torch.zeros(Bsz, device="cuda")

        buf = lambda n, t=torch.bfloat16: torch.empty((Bsz, n), dtype=t, device="cuda")
        codes, scale, qkv, o, y, logits, number = buf(d, torch.int8), torch.empty(Bsz, device="cuda"), buf(nqkv), buf(h * kp), buf(d), buf(V), torch.empty(Bsz, device="cuda")
        codes_o = buf(h * kp, torch.int8)
        top_p = torch.full((Bsz,), 0.9, device="cuda")

        def step(cache, token, prob):
            cache.lens.add_(1)
            x = emb[token.long()]
            own.ecospa_contract_quant(*own.ecospa_quant_rows(x, codes, scale), *weights[0], out=qkv)
            own.ecospa_quant_cache_append(cache, qkv)
            own.ecospa_quant_cache_attn(cache, qkv[:, :h * kp], o)
            own.ecospa_contract_quant(*own.ecospa_quant_rows(o, codes_o, scale), *weights[1], out=y)
            own.ecospa_contract_quant(*own.ecospa_quant_rows(y, codes, scale), *weights[2], out=logits)
            own.ecospa_sample(logits, number, top_p=top_p, token=token, prob=prob)

        eager, want = fresh(), []
        for i in range(7):
            number.copy_(u[i])
            step(*eager)
            want.append((eager[1].clone(), eager[2].clone(), logits.clone()))
        other = fresh()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        number.copy_(u[0])
        with torch.cuda.graph(graph, stream=stream):
            step(*other)
        for i in range(7):
            number.copy_(u[i])
            graph.replay()
            assert torch.equal(other[1], want[i][0]) and torch.equal(other[2], want[i][1]) and torch.equal(logits, want[i][2]), i
            emb.sum().item()                                 # the program's own work between the replays
        assert torch.equal(eager[0].k.view(torch.uint8), other[0].k.view(torch.uint8)) and torch.equal(eager[0].v_scale, other[0].v_scale)
        torch.cuda.synchronize()


def test_the_command_runs_with_8_bits(ctx, capsys):
    main(["--layers", "1", "--batch", "4", "--prefix", "100", "--prompt", "7", "--steps", "12", "--cache-block", "32", "--quant-weights", "--top-p", "0.9"])
    out = capsys.readouterr().out
    assert '"tokens_per_s"' in out and '"int8"' in out and "e4m3" in out
