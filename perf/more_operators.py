"""What serving a coupled-sparse model in eight bits asks of the library, for timing and for comparing outputs.

Kinds of cases:
  linear   a projection whose weights are held in 8-bit integers with a scale for each output channel: the rows of the activations are
           brought to 8 bits with a scale for each token, multiplied, scaled back, with the bias and the activation behind it
  append   the new tokens of B requests after the projection: queries and keys turned by the angles of the kept rotary blocks at each
           request's own position, keys and values put into caches of 8-bit floats (e4m3) with a scale for each block of tokens and head
  attn     attention of L new tokens a request over its own 8-bit cache (ragged lengths up to `own`); with `prefix` the result over the
           tokens that all requests share, computed before, is joined in
  sample   a token drawn for every row of logits by a given random number, after temperature, top-k, top-p and min-p
`own` (the module's name) says whether run() calls the library or computes the same in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

GPT2M = {"h": 16, "h_kv": 16, "kq": 32, "kv": 32}          # half-kept heads of the benchmark's 16-head layer
LLAMA1B = {"h": 32, "h_kv": 32, "kq": 32, "kv": 32}        # half-kept heads of its 32-head layer
DENSE = {"h": 32, "h_kv": 8, "kq": 64, "kv": 64}           # whole heads of 64 dims, four query heads a key/value head
WIDE = {"h": 32, "h_kv": 32, "kq": 96, "kv": 128}          # heads of 128 dims, some rotary blocks removed


def listed():
    return [
        # one new token of one chat through the 16-head layer's output projection, half of its heads' dims kept: nothing but latency
        {"name": "linear_token", "kind": "linear", "T": 1, "N": 1024, "K": 512, "act": "none", "bias": True},
        # a step of a batch through the gated FFN's first matrix of the 32-head layer, half of its units kept
        {"name": "linear_batch", "kind": "linear", "T": 64, "N": 5504, "K": 2048, "act": "swiglu", "bias": False},
        # a step of a batch onto the vocabulary of the stack workloads: the weights have to come from memory
        {"name": "linear_vocab", "kind": "linear", "T": 32, "N": 32000, "K": 2048, "act": "none", "bias": False},
        # the prompts of a batch, an odd number of tokens, through the gated FFN's first matrix
        {"name": "linear_prompts", "kind": "linear", "T": 16 * 509, "N": 5504, "K": 2048, "act": "swiglu", "bias": False},
        # one new token of four chats into their caches
        {"name": "append_token", "kind": "append", **GPT2M, "B": 4, "L": 1, "cap": 1000, "block": 32, "rope": False},
        # the prompts of a batch behind what the caches hold, blocks begun by earlier tokens among them
        {"name": "append_prompts", "kind": "append", **DENSE, "B": 32, "L": 509, "cap": 1024, "block": 64, "rope": True},
        # a single chat
        {"name": "attn_one", "kind": "attn", **LLAMA1B, "B": 1, "L": 1, "own": 1000, "cap": 1024, "block": 32, "prefix": False},
        # a batch of chats with long histories, shared key/value heads
        {"name": "attn_batch", "kind": "attn", **DENSE, "B": 64, "L": 1, "own": 16384, "cap": 16384, "block": 64, "prefix": False},
        # a few drafted tokens a request are checked at once behind a shared prefix, unequal kept widths, odd lengths
        {"name": "attn_drafts", "kind": "attn", **WIDE, "B": 12, "L": 5, "own": 4999, "cap": 5001, "block": 16, "prefix": True},
        # the prompts of a batch over caches that hold earlier turns
        {"name": "attn_prompts", "kind": "attn", **DENSE, "B": 8, "L": 509, "own": 4096, "cap": 4096, "block": 128, "prefix": False},
        # one chat, the vocabulary of the stack workloads
        {"name": "sample_one", "kind": "sample", "B": 1, "V": 32000, "k": 50, "p": True, "min": False, "f32": False},
        # a large batch on a large vocabulary, sets of thousands of tokens kept
        {"name": "sample_large", "kind": "sample", "B": 256, "V": 131072, "k": 0, "p": True, "min": True, "f32": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "append", "attn", "attn", "sample"))
    if kind == "sample":
        return {"kind": kind, "B": _log(rng, 1, 256), "V": _log(rng, 100, 131072), "k": rng.choice((0, 1, _log(rng, 2, 2000))), "p": rng.random() < 0.6,
                "min": rng.random() < 0.4, "f32": rng.random() < 0.5}
    if kind == "linear":
        T, N, K = rng.choice((_log(rng, 1, 64), _log(rng, 1, 8144))), 16 * _log(rng, 2, 2000), 16 * _log(rng, 4, 700)
        T = max(1, min(T, 8144 * 5504 * 2048 // (N * K)))
        return {"kind": kind, "T": T, "N": N, "K": K, "act": rng.choice(("none", "none", "gelu", "swiglu")), "bias": rng.random() < 0.5}
    h, h_kv = rng.choice(((16, 16), (32, 32), (32, 8), (16, 4), (6, 6), (32, 4), (24, 3)))
    heads = {"h": h, "h_kv": h_kv, "kq": 16 * rng.randint(1, 8), "kv": 16 * rng.randint(1, 8)}
    width, block = heads["kq"] + heads["kv"], rng.choice((16, 32, 64, 128))
    if kind == "append":
        L, B = rng.choice((1, 1, _log(rng, 2, 512))), _log(rng, 1, 64)
        B = max(1, min(B, 32 * 509 * 40 * 128 // (L * (h + h_kv) * width)))
        return {"kind": kind, **heads, "B": B, "L": L, "cap": L + _log(rng, 1, 512), "block": block, "rope": rng.random() < 0.7}
    L = rng.choice((1, 1, 1, rng.randint(2, 8), _log(rng, 9, 512)))
    B, length = _log(rng, 1, 64), L - 1 + _log(rng, 1, 16384)
    B = max(1, min(B, 8 * 509 * 32 * 4096 * 128 // (L * h * length * max(width, 128)), 64 * 8 * 16384 * 128 // (h_kv * length * width)))
    return {"kind": kind, **heads, "B": B, "L": L, "own": length, "cap": length + rng.randint(0, 100), "block": block, "prefix": rng.random() < 0.3}


def _lens(case):
    """Lengths of the caches, new tokens among them: the longest, and the others between a third of it and all of it."""
    top, least = case["own"], max(case.get("L", 1), case["own"] // 3)
    return [top - (i * 7919 % (top - least + 1)) for i in range(case["B"])]


def _visible(case):
    """Pairs of a query and a key that it sees."""
    L = case["L"]
    return sum(L * (n - L) + L * (L + 1) // 2 for n in _lens(case))


def work(case):
    k = case["kind"]
    if k == "linear":
        T, N, K = case["T"], case["N"], case["K"]
        return {"bytes": 2 * T * K + N * K + 4 * N + 2 * T * (N // 2 if case["act"] == "swiglu" else N) + (2 * N if case["bias"] else 0), "flops": 2 * T * N * K}
    if k == "sample":
        n = case["B"] * case["V"]
        return {"bytes": n * (4 if case["f32"] else 2) + 24 * case["B"], "flops": 6 * n}
    h, h_kv, kq, kv, B, L = (case[n] for n in ("h", "h_kv", "kq", "kv", "B", "L"))
    T = B * L
    if k == "append":
        turned = T * (h + h_kv) * kq if case["rope"] else T * h_kv * kq
        queries = 2 * T * h * kq if case["rope"] else 0
        return {"bytes": 2 * (turned + T * h_kv * kv) + queries + T * h_kv * (kq + kv) + (4 * T * h_kv * kq if case["rope"] else 0),
                "flops": 3 * turned + 2 * T * h_kv * (kq + kv)}
    keys, prior = sum(_lens(case)), T * h * (2 * kv + 4) if case["prefix"] else 0
    return {"bytes": h_kv * keys * (kq + kv) + 8 * h_kv * (keys // case["block"]) + 2 * T * h * (kq + kv) + 4 * T * h + prior,
            "flops": 2 * h * (kq + kv) * _visible(case)}


# ---- inputs --------------------------------------------------------------------------------------------------------------------------
def _scale_of(top):
    """The least power of two that brings `top` into the range of the 8-bit floats (their largest is 448)."""
    m, e = torch.frexp(top.float() / 448.0)                # top / 448 = m 2^e, m in [1/2, 1)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.ldexp(torch.ones_like(m), e.clamp(min=-100)).masked_fill(top == 0, 2.0 ** -100)


def _to_blocks(x, block):
    """[B, h_kv, cap, d] -> 8-bit values and the scales of its blocks."""
    B, H, cap, d = x.shape
    n = (cap + block - 1) // block
    pad = torch.nn.functional.pad(x.float(), (0, 0, 0, n * block - cap)).view(B, H, n, block, d)
    s = _scale_of(pad.abs().amax((3, 4)))
    return (pad / s[..., None, None]).view(B, H, n * block, d)[:, :, :cap].to(torch.float8_e4m3fn).contiguous(), s.contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    uni = lambda *s: torch.rand(*s, device="cuda", generator=gen)
    ints = lambda hi, *s: torch.randint(0, hi, s, device="cuda", generator=gen, dtype=torch.int32)
    st = {"case": case}
    if case["kind"] == "linear":
        T, N, K = case["T"], case["N"], case["K"]
        # normalised activations, a few channels larger than the others; weights of any scale, brought to 8 bits once
        st["x"] = (rnd(T, K) * torch.exp(0.5 * rnd(K))).bfloat16()
        w = rnd(N, K) * (0.02 * torch.exp(0.3 * rnd(N, 1)))
        st["sw"] = w.abs().amax(1) / 127.0
        st["w"] = torch.round(w / st["sw"][:, None]).to(torch.int8)
        st["bias"] = (0.1 * rnd(N)).bfloat16() if case["bias"] else None
        st["y"] = torch.zeros(T, N // 2 if case["act"] == "swiglu" else N, device="cuda", dtype=torch.bfloat16)
        return st
    B = case["B"]
    if case["kind"] == "sample":
        V = case["V"]
        pitch = (V + 63) // 64 * 64                        # rows of a projection onto a padded vocabulary
        x = (1.5 + 2.0 * uni(B, 1)) * rnd(B, pitch)        # some rows are sure of their next token, some are not
        x = x.masked_fill((uni(B, pitch) < 0.3) & (uni(B, 1) < 0.3), -math.inf)        # and some were masked by a grammar
        x[:, V // 2] = 1.0
        st["logits"] = x.to(torch.float32 if case["f32"] else torch.bfloat16)[:, :V]
        st["u"] = uni(B)
        st["temp"] = (0.5 + uni(B)).masked_fill(uni(B) < 0.1, 0.0)        # 0: the best token
        st["top_k"] = (1 + ints(case["k"], B)) if case["k"] else None
        st["top_p"] = 0.5 + 0.5 * uni(B) if case["p"] else None
        st["min_p"] = 0.1 * uni(B) * (uni(B) < 0.7) if case["min"] else None
        st["token"], st["prob"] = torch.zeros(B, device="cuda", dtype=torch.int32), torch.zeros(B, device="cuda")
        return st
    h, h_kv, kq, kv, cap, L, block = (case[n] for n in ("h", "h_kv", "kq", "kv", "cap", "L", "block"))
    # keys and values scatter around a mean of their head, as trained ones do, and tokens differ in their size
    size = lambda *s: torch.exp(0.5 * rnd(*s, 1))
    st["k"], st["k_scale"] = _to_blocks(rnd(B, h_kv, cap, kq) * size(B, h_kv, cap) + 0.5 * rnd(h_kv, 1, kq), block)
    st["v"], st["v_scale"] = _to_blocks(rnd(B, h_kv, cap, kv) * size(B, h_kv, cap) + 0.5 * rnd(h_kv, 1, kv), block)
    if case["kind"] == "append":
        st["qkv"] = (rnd(B * L, (h + h_kv) * kq + h_kv * kv) * size(B * L)).bfloat16()
        st["lens"] = L + ints(cap - L + 1, B)
        st["pos"] = (st["lens"] - L + ints(1000, 1)).int()
        st["q"] = torch.zeros(B * L, h * kq, device="cuda", dtype=torch.bfloat16)
        if case["rope"]:                                   # kept rotary blocks differ from head to head
            blocks = uni(h_kv, 64).topk(kq // 2, dim=1).indices.sort(dim=1).values
            angle = torch.arange(cap + 1000, device="cuda", dtype=torch.float64)[None, :, None] * (10000.0 ** (-2.0 * blocks.double() / 128))[:, None]
            st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        return st
    st["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[torch.randperm(B, device="cuda", generator=gen)]
    st["q"] = rnd(B * L, h * kq).bfloat16()
    st["o"], st["lse"] = torch.zeros(B * L, h * kv, device="cuda", dtype=torch.bfloat16), torch.zeros(B, h, L, device="cuda")
    if case["prefix"]:                                     # what the attention over a prefix of a few thousand tokens leaves
        st["o_in"], st["lse_in"] = (0.5 * rnd(B * L, h * kv)).bfloat16(), 8.0 + 0.5 * rnd(B, h, L)
    return st


def _scale(case):
    return 1.0 / math.sqrt(64.0 if case["kq"] <= 64 else 128.0)      # of the head before dims were removed


# ---- the library's calls -----------------------------------------------------------------------------------------------------------------
_context = None


def _own(st):
    global _context
    from paper_2511_11641_amd import binding as B
    if _context is None:
        _context = B.Context("cuda:0")
    ctx, case = _context, st["case"]
    if case["kind"] == "linear":
        act = {"none": None, "gelu": B.ACT_GELU_ERF, "swiglu": B.ACT_SWIGLU}[case["act"]]
        x, s = ctx.ecospa_quant_rows(st["x"])
        return {"y": ctx.ecospa_contract_quant(x, s, st["w"], st["sw"], bias=st["bias"], act=act, out=st["y"])}
    if case["kind"] == "sample":
        ctx.ecospa_sample(st["logits"], st["u"], temperature=st["temp"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"], token=st["token"], prob=st["prob"])
        return {"token": st["token"], "prob": st["prob"]}
    if "cache" not in st:                                  # a program keeps its cache object beside the cache
        st["cache"] = B.QuantCache(st["k"], st["v"], st["k_scale"], st["v_scale"], st["lens"], case["h"], _scale(case), case["block"],
                                 own_max=case.get("own", case["cap"]))
    if case["kind"] == "append":
        rope = (st["cos"], st["sin"]) if case["rope"] else None
        ctx.ecospa_quant_cache_append(st["cache"], st["qkv"], st["pos"], rope=rope, q=st["q"] if rope else None)
        return _cache_out(st)
    ctx.ecospa_quant_cache_attn(st["cache"], st["q"], st["o"], lse=st["lse"], o_in=st.get("o_in"), lse_in=st.get("lse_in"))
    return {"o": st["o"], "lse": st["lse"]}


def _cache_out(st):
    return {"k": st["k"], "v": st["v"], "k_scale": st["k_scale"], "v_scale": st["v_scale"], **({"q": st["q"]} if st["case"]["rope"] else {})}


# ---- the plain forms ---------------------------------------------------------------------------------------------------------------------
def run(st):
    return _own(st) if own else {"linear": _linear, "append": _append, "attn": _attn, "sample": _sample}[st["case"]["kind"]](st)


def _linear(st):
    c, x = st["case"], st["x"].float()
    s = x.abs().amax(1, keepdim=True) / 127.0
    q = torch.round(x / s.masked_fill(s == 0, 1.0))
    y = torch.matmul(q, st["w"].float().t()) * s * st["sw"]
    if c["bias"]:
        y = y + st["bias"].float()
    if c["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if c["act"] == "swiglu":                               # columns are (gate, up) pairs
        y = y[:, 0::2] / (1.0 + torch.exp(-y[:, 0::2])) * y[:, 1::2]
    return {"y": y.bfloat16()}


def _turn(x, cos, sin):
    x0, x1 = x[..., 0::2].float(), x[..., 1::2].float()
    return torch.stack((x0 * cos - x1 * sin, x0 * sin + x1 * cos), dim=-1).reshape(x.shape)


def _append(st):
    c = st["case"]
    B, L, h, h_kv, kq, kv = (c[n] for n in ("B", "L", "h", "h_kv", "kq", "kv"))
    q, k, v = st["qkv"].view(B, L, -1).split((h * kq, h_kv * kq, h_kv * kv), dim=2)
    k, v = k.reshape(B, L, h_kv, kq), v.reshape(B, L, h_kv, kv)
    if c["rope"]:
        at = st["pos"].long()[:, None] + torch.arange(L, device="cuda")
        cos, sin = st["cos"][:, at].permute(1, 2, 0, 3), st["sin"][:, at].permute(1, 2, 0, 3)        # [B, L, h_kv, kq / 2]
        st["q"].copy_(_turn(q.reshape(B, L, h, kq), cos.repeat_interleave(h // h_kv, 2), sin.repeat_interleave(h // h_kv, 2)).reshape(B * L, h * kq))
        k = _turn(k, cos, sin).bfloat16()
    _put(c, st["lens"].long(), st["k"], st["k_scale"], k)
    _put(c, st["lens"].long(), st["v"], st["v_scale"], v)
    return _cache_out(st)


def _put(c, lens, codes, scales, new):
    """The rows new [B, L, h_kv, d] behind the rows that the caches hold: every block that they fall into gets a scale that covers them as
    well, never a smaller one than its earlier rows have, and those rows are brought to it."""
    B, L, block, cap = c["B"], c["L"], c["block"], c["cap"]
    first = lens - L
    base = first // block * block                          # row where the first of the blocks begins
    W = (L + 2 * block - 2) // block * block               # rows of the blocks, at most
    row = base[:, None] + torch.arange(W, device="cuda")   # [B, W]
    t = row - first[:, None]
    old, fresh = t < 0, (t >= 0) & (t < L)
    b, at = torch.arange(B, device="cuda")[:, None], row.clamp(max=cap - 1)
    n = scales.shape[2]
    blk = base[:, None] // block + torch.arange(W // block, device="cuda")
    before = scales[b, :, blk.clamp(max=n - 1)]            # [B, blocks, h_kv]
    x = new[b, t.clamp(0, L - 1)].float().masked_fill(~fresh[..., None, None], 0.0)
    x = x + (codes[b, :, at].float() * before.repeat_interleave(block, 1)[..., None]).masked_fill(~old[..., None, None], 0.0)
    top = x.abs().view(B, W // block, block, *x.shape[2:]).masked_fill(old.view(B, -1, block)[..., None, None], 0.0).amax((2, 4))
    some = old.view(B, -1, block).any(2)[..., None]        # blocks with earlier rows
    s = torch.maximum(_scale_of(top), before.masked_fill(~some, 0.0))
    y = (x / s.repeat_interleave(block, 1)[..., None]).to(torch.float8_e4m3fn)
    written = (old | fresh) & (row < cap)
    i, j = written.nonzero(as_tuple=True)
    codes.view(torch.uint8)[i, :, row[i, j]] = y.view(torch.uint8)[i, j]
    i, j = fresh.view(B, -1, block).any(2).nonzero(as_tuple=True)
    scales[i, :, blk[i, j]] = s[i, j]


def _attn(st):
    c = st["case"]
    B, L, h, h_kv, kq, kv, S, block = (c[n] for n in ("B", "L", "h", "h_kv", "kq", "kv", "own", "block"))
    g = h // h_kv
    values = lambda x, s: x[:, :, :S].float().mul_(s.repeat_interleave(block, 2)[:, :, :S, None])
    q = st["q"].float().view(B, L, h_kv, g, kq).permute(0, 2, 1, 3, 4).reshape(B, h_kv, L * g, kq)
    s = torch.matmul(q, values(st["k"], st["k_scale"]).transpose(2, 3).contiguous()).mul_(_scale(c)).view(B, h_kv, L, g, S)
    n = st["lens"][:, None] - L + 1 + torch.arange(L, device="cuda")                                # keys that a query sees
    s = s.masked_fill_((torch.arange(S, device="cuda") >= n[:, :, None])[:, None, :, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    if c["prefix"]:
        before = st["lse_in"].view(B, h_kv, g, L).transpose(2, 3)[..., None]
        top = torch.maximum(top, before)
    ref = top.masked_fill(top == -math.inf, 0.0)
    s = s.sub_(ref).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, h_kv, L * g, S), values(st["v"], st["v_scale"])).view(B, h_kv, L, g, kv)
    if c["prefix"]:
        share = (before - ref).exp()
        total = total + share
        o = o + share * st["o_in"].float().view(B, L, h_kv, g, kv).transpose(1, 2)
    o = o * torch.where(total > 0, 1.0 / total, 0.0)
    return {"o": o.transpose(1, 2).reshape(B * L, h * kv).bfloat16(), "lse": (ref + total.log())[..., 0].transpose(2, 3).reshape(B, h, L)}


def _sample(st):
    x = st["logits"].float()
    B, V = x.shape
    # which tokens are drawn lies next to borders: in 64 bits
    temp = st["temp"].double()[:, None]
    best = x.amax(1, keepdim=True)
    first = torch.where(x == best, torch.arange(V, device="cuda"), V).amin(1)
    w = torch.exp((x.double() - best.double()) / temp.masked_fill(temp == 0, 1.0))
    order = x.sort(dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    keep = torch.ones_like(ws, dtype=torch.bool)
    if st["top_k"] is not None:
        keep &= torch.arange(V, device="cuda") < st["top_k"].long()[:, None]
        ws = ws * keep
    if st["top_p"] is not None:
        cum = ws.cumsum(1)
        ahead = torch.nn.functional.pad(cum[:, :-1], (1, 0))
        keep &= ahead < st["top_p"].double()[:, None] * cum[:, -1:]
    if st["min_p"] is not None:
        keep &= ws >= st["min_p"].double()[:, None]
    w = w * torch.zeros_like(keep).scatter_(1, order, keep)
    cum = w.cumsum(1)
    token = (cum <= st["u"].double()[:, None] * cum[:, -1:]).sum(1)
    prob = w.gather(1, token[:, None])[:, 0] / cum[:, -1]
    greedy = temp[:, 0] == 0
    return {"token": torch.where(greedy, first, token).int(), "prob": prob.masked_fill(greedy, 1.0).float()}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear":
        x, rows = st["x"].double(), []
        gelu = lambda z: z * torch.special.ndtr(z)
        for part in x.split(1024):
            # the codes are whole numbers next to borders that 32 bits decide
            s = (part.float().abs().amax(1) / 127.0).double()
            q = torch.round((part.float() / s.float().masked_fill(s == 0, 1.0)[:, None])).double()
            y = (q @ st["w"].double().t().contiguous()) * s[:, None] * st["sw"].double()
            y = y + st["bias"].double() if case["bias"] else y
            if case["act"] == "swiglu":
                gate, up = y.view(y.shape[0], -1, 2).unbind(2)
                y = torch.sigmoid(gate) * gate * up
            rows.append(gelu(y) if case["act"] == "gelu" else y)
        return {"y": torch.cat(rows)}
    B = case["B"]
    if kind == "sample":
        host = lambda n, off: [off] * B if st[n] is None else st[n].cpu().double().tolist()
        top_k, top_p, min_p, probs = host("top_k", case["V"]), host("top_p", 1.0), host("min_p", 0.0), []
        temp, u = st["temp"].cpu().double().tolist(), st["u"].cpu().double().tolist()
        for b in range(B):
            x = st["logits"][b].cpu().double().numpy()
            if temp[b] == 0.0:
                probs.append(1.0)
                continue
            rank = np.lexsort((np.arange(x.size), -x))[:int(top_k[b])]
            w = np.exp((x[rank] - x[rank[0]]) / temp[b])
            behind = np.searchsorted(np.cumsum(w), top_p[b] * w.sum()) + 1
            kept = rank[:behind][w[:behind] >= min_p[b]]
            kept.sort()
            w = np.exp((x[kept] - x[rank[0]]) / temp[b])
            i = min(int(np.searchsorted(np.cumsum(w), u[b] * w.sum(), side="right")), kept.size - 1)
            probs.append(float(w[i] / w.sum()))
        return {"token": None, "prob": np.array(probs)}
    h, h_kv, kq, kv, L, block = (case[n] for n in ("h", "h_kv", "kq", "kv", "L", "block"))
    lens, g = st["lens"].tolist(), h // h_kv
    if kind == "append":
        # the 8-bit values as real numbers, not rounded
        rows = st["qkv"].double().view(B, L, -1)
        q, key, val = rows[..., :h * kq], rows[..., h * kq:(h + h_kv) * kq], rows[..., (h + h_kv) * kq:]
        q, key, val = q.reshape(B, L, h, kq), key.reshape(B, L, h_kv, kq), val.reshape(B, L, h_kv, kv)
        turned, held = torch.empty_like(q), {n: st[n].double() for n in ("k", "v", "k_scale", "v_scale")}
        for b in range(B):
            kb = key[b]
            if case["rope"]:
                p = int(st["pos"][b])
                z = torch.complex(st["cos"][:, p:p + L].double(), st["sin"][:, p:p + L].double()).transpose(0, 1)      # [L, h_kv, kq / 2]
                kb = torch.view_as_real(torch.view_as_complex(kb.reshape(L, h_kv, -1, 2)) * z).reshape(L, h_kv, kq)
                zq = z[:, torch.arange(h, device="cuda") // g]
                turned[b] = torch.view_as_real(torch.view_as_complex(q[b].reshape(L, h, -1, 2)) * zq).reshape(L, h, kq)
            lo, hi = lens[b] - L, lens[b]
            for name, x in (("k", kb.bfloat16().double()), ("v", val[b])):
                codes, scales = held[name][b], held[name + "_scale"][b]
                for i in range(lo // block, (hi - 1) // block + 1):
                    a, e = max(lo, i * block), min(hi, (i + 1) * block)
                    least = torch.ceil(torch.log2(x[a - lo:e - lo].abs().amax((0, 2)) / 448.0)).clamp(min=-100.0)
                    s = torch.maximum(torch.exp2(least), scales[:, i]) if a > i * block else torch.exp2(least)
                    codes[:, i * block:a] *= (scales[:, i] / s)[:, None, None]
                    codes[:, a:e] = x[a - lo:e - lo].transpose(0, 1) / s[:, None, None]
                    scales[:, i] = s
        return {**held, **({"q": turned.reshape(B * L, h * kq)} if case["rope"] else {})}
    if 2 * h * (kq + kv) * _visible(case) > 4e12:
        return None
    o = torch.zeros(B, L, h, kv, device="cuda", dtype=torch.float64)
    lse = torch.zeros(B, h, L, device="cuda", dtype=torch.float64)
    q = st["q"].double().view(B, L, h, kq)
    for b in range(B):
        n = lens[b]
        blk = torch.arange(n, device="cuda") // block
        for j in range(h_kv):
            heads = slice(j * g, (j + 1) * g)
            keys, vals = (st[x][b, j, :n].double() * st[x + "_scale"][b, j].double()[blk, None] for x in ("k", "v"))
            s = q[b, :, heads].transpose(0, 1).reshape(-1, kq).mul(_scale(case)) @ keys.T                  # [group * L, n]
            late = torch.arange(n, device="cuda") >= n - L + 1 + torch.arange(L, device="cuda")[:, None]
            s = s.view(-1, L, n).masked_fill(late, -math.inf)
            own_z = torch.logsumexp(s, -1)
            z = own_z
            if case["prefix"]:
                before = st["lse_in"][b, heads].double()
                z = torch.logaddexp(own_z, before)
            out = torch.exp(s - z[..., None]) @ vals
            if case["prefix"]:
                out = out + torch.exp(before - z)[..., None] * st["o_in"].double().view(B, L, h, kv)[b, :, heads].transpose(0, 1)
            lse[b, heads], o[b, :, heads] = z, out.transpose(0, 1)
    return {"o": o.reshape(B * L, h * kv), "lse": lse}
