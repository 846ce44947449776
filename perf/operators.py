"""What serving a coupled-sparse model token by token asks of the library, for timing and for comparing outputs.

Kinds of cases (compact heads: h query heads on h_kv key/value heads, kq and kv kept dims a head):
  append   the new tokens of B requests after the projection: queries and keys turned by the angles of the kept rotary
           blocks at each request's own position, keys and values put into the requests' own caches
  attn     attention of L new tokens a request over a prefix of P tokens that all requests share and over the request's own
           cache (ragged lengths up to `own`); with `weights` the probability that every own key received is accumulated
  evict    own caches cut down to `keep` keys: the last `recent` and, of the others, those with the most accumulated weight
  logits   penalties for tokens of the history, per-token biases, temperature and grammar masks on logits; the best token
           and the log-sum-exp of every row
`own` (the module's name) says whether run() calls the library or computes the same in elementary torch operations.
"""
import math

import torch

own = False

GPT2M = {"h": 16, "h_kv": 16, "kq": 32, "kv": 32}          # half-kept heads of the benchmark's 16-head layer
LLAMA1B = {"h": 32, "h_kv": 32, "kq": 32, "kv": 32}        # half-kept heads of its 32-head layer
DENSE = {"h": 32, "h_kv": 8, "kq": 64, "kv": 64}           # whole heads of 64 dims, four query heads a key/value head
WIDE = {"h": 32, "h_kv": 32, "kq": 96, "kv": 128}          # heads of 128 dims, some rotary blocks removed


def listed():
    return [
        # one new token of four chats: nothing but latency
        {"name": "append_token", "kind": "append", **GPT2M, "B": 4, "L": 1, "cap": 1024, "rope": False},
        # the prompts of a batch behind their common prefix go into the cache in one call
        {"name": "append_prompts", "kind": "append", **DENSE, "B": 32, "L": 509, "cap": 1024, "rope": True},
        # a single chat with a short system prompt: the least a decoder asks for
        {"name": "attn_one", "kind": "attn", **GPT2M, "B": 1, "L": 1, "P": 61, "own": 33, "cap": 256, "weights": False},
        # a batch of chats on a system prompt of a few thousand tokens
        {"name": "attn_batch", "kind": "attn", **LLAMA1B, "B": 32, "L": 1, "P": 4096, "own": 500, "cap": 1024, "weights": True},
        # many questions on one long document, shared key/value heads, weights kept for the eviction
        {"name": "attn_document", "kind": "attn", **DENSE, "B": 64, "L": 1, "P": 32768, "own": 2048, "cap": 2048, "weights": True},
        # a few drafted tokens a request are checked at once, unequal kept widths, odd lengths
        {"name": "attn_drafts", "kind": "attn", **WIDE, "B": 12, "L": 5, "P": 8191, "own": 300, "cap": 512, "weights": False},
        # the prompts of a batch over the prefix they share
        {"name": "attn_prompts", "kind": "attn", **DENSE, "B": 16, "L": 509, "P": 8192, "own": 509, "cap": 1024, "weights": False},
        # a few chats that reached their limit
        {"name": "evict_few", "kind": "evict", **GPT2M, "B": 3, "cap": 1000, "own": 1000, "keep": 512, "recent": 64},
        # every cache of a batch
        {"name": "evict_batch", "kind": "evict", **DENSE, "B": 32, "cap": 8192, "own": 8192, "keep": 2048, "recent": 256},
        # one chat, the vocabulary of the stack workloads
        {"name": "logits_one", "kind": "logits", "B": 1, "V": 32000, "hist": 61, "bias": 0, "masks": 0, "f32": False},
        # a batch on the other vocabulary, odd width of rows with padding behind them, biases and masks
        {"name": "logits_batch", "kind": "logits", "B": 64, "V": 50257, "hist": 2048, "bias": 37, "masks": 3, "f32": False},
        # a large batch on a large vocabulary with long histories
        {"name": "logits_large", "kind": "logits", "B": 256, "V": 131072, "hist": 8192, "bias": 300, "masks": 16, "f32": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "attn", "attn", "evict", "logits"))
    if kind == "logits":
        B, V, hist = _log(rng, 1, 256), _log(rng, 1000, 131072), _log(rng, 1, 8192)
        return {"kind": kind, "B": B, "V": V, "hist": hist, "bias": rng.choice((0, 1, _log(rng, 2, 300))), "masks": rng.choice((0, 1, _log(rng, 1, 16))),
                "f32": rng.random() < 0.5}
    h, h_kv = rng.choice(((16, 16), (32, 32), (32, 8), (16, 4), (6, 6), (32, 4), (24, 3)))
    heads = {"h": h, "h_kv": h_kv, "kq": 16 * rng.randint(1, 8), "kv": 16 * rng.randint(1, 8)}
    width = heads["kq"] + heads["kv"]
    if kind == "append":
        L, B = rng.choice((1, 1, _log(rng, 2, 512))), _log(rng, 1, 64)
        B = max(1, min(B, 32 * 509 * 48 * 64 // (L * (h + h_kv) * width)))
        return {"kind": kind, **heads, "B": B, "L": L, "cap": L + _log(rng, 1, 512), "rope": rng.random() < 0.7}
    if kind == "evict":
        length, B = _log(rng, 20, 8192), _log(rng, 1, 32)
        B = max(1, min(B, 32 * 8 * 8192 * 128 // (h_kv * length * width)))
        keep = max(1, int(length * rng.uniform(0.2, 1.1)))
        return {"kind": kind, **heads, "B": B, "cap": length + rng.randint(0, 40), "own": length, "keep": keep, "recent": int(keep * rng.uniform(0, 0.5))}
    L = rng.choice((1, 1, 1, rng.randint(2, 8), _log(rng, 9, 512)))
    B, P, length = _log(rng, 1, 64), rng.choice((0, _log(rng, 1, 32768), _log(rng, 500, 32768))), L - 1 + _log(rng, 1, 2048)
    B = max(1, min(B, 16 * 509 * 32 * 8704 * 128 // (L * h * (P + length) * max(width, 128))))
    return {"kind": kind, **heads, "B": B, "L": L, "P": P, "own": length, "cap": length + rng.randint(0, 100), "weights": rng.random() < 0.5}


def _lens(case):
    """Lengths of the own caches, new tokens among them: the longest, and the others between a third of it and all of it."""
    top, least = case["own"], max(case.get("L", 1), case["own"] // 3)
    return [top - (i * 7919 % (top - least + 1)) for i in range(case["B"])]


def _visible(case):
    """Pairs of a query and an own key that it sees."""
    L = case["L"]
    return sum(L * (n - L) + L * (L + 1) // 2 for n in _lens(case))


def work(case):
    k = case["kind"]
    if k == "logits":
        size = 4 if case["f32"] else 2
        n = case["B"] * case["V"]
        return {"bytes": 2 * n * size + 4 * case["B"] * (case["hist"] + 2 * case["bias"]) + case["masks"] * case["V"] // 8 + 8 * case["B"], "flops": 6 * n}
    h, h_kv, kq, kv, B = (case[n] for n in ("h", "h_kv", "kq", "kv", "B"))
    if k == "append":
        T = B * case["L"]
        turned = T * (h + h_kv) * kq if case["rope"] else T * h_kv * kq
        return {"bytes": 2 * 2 * (turned + T * h_kv * kv) + (4 * T * h_kv * kq if case["rope"] else 0), "flops": 3 * turned if case["rope"] else 0}
    if k == "evict":
        kept = sum(min(n, case["keep"]) for n in _lens(case))
        return {"bytes": h_kv * (4 * sum(_lens(case)) + kept * (4 * (kq + kv) + 8)), "flops": 0}
    T, keys = B * case["L"], sum(_lens(case))
    bytes_ = 2 * (h_kv * (case["P"] + keys) * (kq + kv) + T * h * (kq + kv)) + 4 * T * h + (8 * h_kv * keys if case["weights"] else 0)
    return {"bytes": bytes_, "flops": 2 * h * (kq + kv) * (T * case["P"] + _visible(case))}


# ---- inputs --------------------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    ints = lambda hi, *s: torch.randint(0, hi, s, device="cuda", generator=gen, dtype=torch.int32)
    B, st = case["B"], {"case": case}
    if case["kind"] == "logits":
        V, H = case["V"], case["hist"]
        pitch = (V + 63) // 64 * 64                        # rows of a projection onto a padded vocabulary
        dt = torch.float32 if case["f32"] else torch.bfloat16
        st["logits"] = (2.5 * rnd(B, pitch)).to(dt)[:, :V]
        st["out"] = torch.zeros(B, pitch, device="cuda", dtype=dt)[:, :V]
        # a history repeats itself: tokens of a few hundred, often the same ones
        pool = ints(V, B, max(1, H // 4))
        st["hist"] = pool.gather(1, (torch.rand(B, H, device="cuda", generator=gen).square() * pool.shape[1]).long())
        st["hist_len"] = torch.tensor([H - i * 31 % (H // 2 + 1) for i in range(B)], dtype=torch.int32, device="cuda")
        st["rep"], st["freq"] = 1.0 + 0.3 * rnd(B).abs(), 0.2 * rnd(B).abs()
        st["pres"], st["temp"] = 0.3 * rnd(B).abs(), 0.6 + 0.2 * rnd(B).abs()
        if case["bias"]:
            n = case["bias"]
            st["bias_ids"] = torch.rand(B, V, device="cuda", generator=gen).topk(n, dim=1).indices.int() if B * V < 1 << 26 else \
                ((torch.arange(n, device="cuda", dtype=torch.int32) * (V // n))[None] + ints(V // n, B, n))
            st["bias"] = 2.0 * rnd(B, n)
        if case["masks"]:
            st["mask"] = torch.randint(-(1 << 31), 1 << 31, (case["masks"], (V + 31) // 32), device="cuda", generator=gen).int()
            st["mask_row"] = ints(case["masks"] + 1, B) - 1       # -1: no grammar
        return st
    h, h_kv, kq, kv, cap = (case[n] for n in ("h", "h_kv", "kq", "kv", "cap"))
    # keys and values scatter around a mean of their head, as trained ones do
    keys = lambda *s: (rnd(*s, kq) + 0.5 * rnd(h_kv, 1, kq)).bfloat16()
    values = lambda *s: (rnd(*s, kv) + 0.5 * rnd(h_kv, 1, kv)).bfloat16()
    st["k"], st["v"] = keys(B, h_kv, cap), values(B, h_kv, cap)
    if case["kind"] == "append":
        L = case["L"]
        lens = L + ints(cap - L + 1, B)
        st["qkv"] = rnd(B * L, (h + h_kv) * kq + h_kv * kv).bfloat16()
        st["lens"], st["pos"] = lens, (lens - L + ints(1000, 1)).int()
        st["q"] = torch.zeros(B * L, h * kq, device="cuda", dtype=torch.bfloat16)
        st["w"] = torch.rand(B, h_kv, cap, device="cuda", generator=gen)
        if case["rope"]:                                   # kept rotary blocks differ from head to head
            blocks = torch.rand(h_kv, 64, device="cuda", generator=gen).topk(kq // 2, dim=1).indices.sort(dim=1).values
            angle = torch.arange(cap + 1000, device="cuda", dtype=torch.float64)[None, :, None] * (10000.0 ** (-2.0 * blocks.double() / 128))[:, None]
            st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        return st
    order = torch.randperm(B, device="cuda", generator=gen)
    st["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[order]
    if case["kind"] == "evict":
        # weights as attention leaves them: a few keys hold most, the newest and some others have none yet
        w = torch.exp(1.5 * rnd(B, h_kv, cap)) * (torch.rand(B, h_kv, cap, device="cuda", generator=gen) > 0.1)
        st["w"] = w
        st["k_out"] = torch.zeros(B, h_kv, case["keep"], kq, device="cuda", dtype=torch.bfloat16)
        st["v_out"] = torch.zeros(B, h_kv, case["keep"], kv, device="cuda", dtype=torch.bfloat16)
        st["w_out"] = torch.zeros(B, h_kv, case["keep"], device="cuda")
        st["lens_out"] = torch.zeros(B, device="cuda", dtype=torch.int32)
        st["idx"] = torch.zeros(B, h_kv, case["keep"], device="cuda", dtype=torch.int32)
        return st
    L, P = case["L"], case["P"]
    st["pk"], st["pv"] = keys(h_kv, P), values(h_kv, P)
    st["q"] = rnd(B * L, h * kq).bfloat16()
    st["o"] = torch.zeros(B * L, h * kv, device="cuda", dtype=torch.bfloat16)
    st["lse"] = torch.zeros(B, h, L, device="cuda")
    if case["weights"]:
        alive = torch.arange(cap, device="cuda") < st["lens"][:, None, None]
        st["w"] = torch.rand(B, h_kv, cap, device="cuda", generator=gen) * alive
        st["w_out"] = torch.zeros(B, h_kv, cap, device="cuda")
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
    if case["kind"] == "logits":
        pick, lse = ctx.ecospa_logits_process(st["logits"], out=st["out"], history=st["hist"], history_len=st["hist_len"], repetition=st["rep"],
                                              frequency=st["freq"], presence=st["pres"], temperature=st["temp"], bias_ids=st.get("bias_ids"),
                                              bias=st.get("bias"), mask=st.get("mask"), mask_row=st.get("mask_row"))
        return {"logits": st["out"], "pick": pick, "lse": lse}
    if "cache" not in st:                                  # a program keeps its cache object beside the cache
        st["cache"] = B.KvCache(st["k"], st["v"], st["lens"], case["h"], _scale(case), st.get("pk"), st.get("pv"), own_max=case.get("own", case["cap"]))
    cache = st["cache"]
    if case["kind"] == "append":
        rope = (st["cos"], st["sin"]) if case["rope"] else None
        ctx.ecospa_cache_append(cache, st["qkv"], st["pos"], rope=rope, q=st["q"] if rope else None, weights=st["w"])
        return {"k": st["k"], "v": st["v"], "w": st["w"], **({"q": st["q"]} if rope else {})}
    if case["kind"] == "evict":
        ctx.ecospa_cache_evict(cache, st["w"], case["keep"], case["recent"], st["k_out"], st["v_out"], st["lens_out"], st["w_out"], st["idx"])
        return {n: st[n] for n in ("k_out", "v_out", "w_out", "lens_out", "idx")}
    ctx.ecospa_prefix_attn(cache, st["q"], st["o"], lse=st["lse"], weights=st.get("w"), weights_out=st.get("w_out"))
    return {"o": st["o"], "lse": st["lse"], **({"w": st["w_out"]} if case["weights"] else {})}


# ---- the plain forms ---------------------------------------------------------------------------------------------------------------------
def run(st):
    return _own(st) if own else {"append": _append, "attn": _attn, "evict": _evict, "logits": _logits}[st["case"]["kind"]](st)


def _append(st):
    c = st["case"]
    B, L, h, h_kv, kq, kv = (c[n] for n in ("B", "L", "h", "h_kv", "kq", "kv"))
    q, k, v = st["qkv"].view(B, L, -1).split((h * kq, h_kv * kq, h_kv * kv), dim=2)
    k, v = k.reshape(B, L, h_kv, kq), v.reshape(B, L, h_kv, kv)
    step = torch.arange(L, device="cuda")
    slot, b = (st["lens"].long() - L)[:, None] + step, torch.arange(B, device="cuda")[:, None]
    if c["rope"]:
        at = st["pos"].long()[:, None] + step
        cos, sin = st["cos"][:, at].permute(1, 2, 0, 3), st["sin"][:, at].permute(1, 2, 0, 3)        # [B, L, h_kv, kq / 2]
        st["q"].copy_(_turn(q.reshape(B, L, h, kq), cos.repeat_interleave(h // h_kv, 2), sin.repeat_interleave(h // h_kv, 2)).reshape(B * L, h * kq))
        k = _turn(k, cos, sin).bfloat16()
    st["k"][b, :, slot] = k
    st["v"][b, :, slot] = v
    st["w"][b, :, slot] = 0.0
    return {"k": st["k"], "v": st["v"], "w": st["w"], **({"q": st["q"]} if c["rope"] else {})}


def _turn(x, cos, sin):
    x0, x1 = x[..., 0::2].float(), x[..., 1::2].float()
    return torch.stack((x0 * cos - x1 * sin, x0 * sin + x1 * cos), dim=-1).reshape(x.shape)


def _attn(st):
    c = st["case"]
    B, L, h, h_kv, kq, kv, P, S = (c[n] for n in ("B", "L", "h", "h_kv", "kq", "kv", "P", "own"))
    g, scale = h // h_kv, _scale(c)
    q = st["q"].float().view(B, L, h_kv, g, kq)
    qp = q.permute(2, 0, 1, 3, 4).reshape(h_kv, B * L * g, kq)
    sp = torch.matmul(qp, st["pk"].float().transpose(1, 2).contiguous()).mul_(scale).view(h_kv, B, L, g, P)
    qo = q.permute(0, 2, 1, 3, 4).reshape(B, h_kv, L * g, kq)
    so = torch.matmul(qo, st["k"][:, :, :S].float().transpose(2, 3).contiguous()).mul_(scale).view(B, h_kv, L, g, S).permute(1, 0, 2, 3, 4)
    n = st["lens"][:, None] - L + 1 + torch.arange(L, device="cuda")                                # own keys that a query sees
    so = so.masked_fill(torch.arange(S, device="cuda") >= n[None, :, :, None, None], -math.inf)
    top = so.amax(-1, keepdim=True)
    top = torch.maximum(top, sp.amax(-1, keepdim=True)) if P else top
    ref = top.masked_fill(top == -math.inf, 0.0)
    sp, so = sp.sub_(ref).exp_(), (so - ref).exp_()
    total = sp.sum(-1, keepdim=True) + so.sum(-1, keepdim=True)
    o = torch.matmul(so.permute(1, 0, 2, 3, 4).reshape(B, h_kv, L * g, S), st["v"][:, :, :S].float()).view(B, h_kv, L, g, kv).permute(0, 2, 1, 3, 4)
    o = o + torch.matmul(sp.view(h_kv, B * L * g, P), st["pv"].float()).view(h_kv, B, L, g, kv).permute(1, 2, 0, 3, 4)
    share = torch.where(total > 0, 1.0 / total, 0.0)
    o = o * share.permute(1, 2, 0, 3, 4)
    out = {"o": o.reshape(B * L, h * kv).bfloat16(), "lse": (ref + total.log())[..., 0].permute(1, 0, 3, 2).reshape(B, h, L)}
    if c["weights"]:
        out["w"] = st["w"].clone()
        out["w"][:, :, :S] += (so * share).sum((2, 3)).transpose(0, 1)
    return out


def _evict(st):
    c = st["case"]
    keep, cap = c["keep"], c["cap"]
    j, n = torch.arange(cap, device="cuda"), st["lens"].long()[:, None, None]
    w = st["w"].masked_fill(j >= n - c["recent"], math.inf).masked_fill(j >= n, -math.inf)
    w = torch.nn.functional.pad(w, (0, max(0, keep - cap)), value=-math.inf)
    idx = w.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    idx = idx.masked_fill(idx >= n, w.shape[-1]).sort(dim=-1).values
    alive = torch.arange(keep, device="cuda") < n.clamp(max=keep)
    at = idx.masked_fill(~alive, 0)
    rows = lambda x: (x.gather(2, at[..., None].expand(-1, -1, -1, x.shape[3])) * alive[..., None].to(x.dtype))
    return {"k_out": rows(st["k"]), "v_out": rows(st["v"]), "w_out": st["w"].gather(2, at) * alive, "lens_out": st["lens"].clamp(max=keep),
            "idx": idx.masked_fill(~alive, -1).int()}


def _logits(st):
    c, x = st["case"], st["logits"].float()
    B, V, H = c["B"], c["V"], c["hist"]
    alive = torch.arange(H, device="cuda") < st["hist_len"][:, None]
    count = torch.zeros(B, V, device="cuda").scatter_add_(1, st["hist"].long(), alive.float())
    seen = count > 0
    rep = st["rep"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - st["freq"][:, None] * count - st["pres"][:, None] * seen
    if c["bias"]:
        x = x.scatter_add(1, st["bias_ids"].long(), st["bias"])
    x = x / st["temp"][:, None]
    if c["masks"]:
        v = torch.arange(V, device="cuda")
        bits = (st["mask"][:, v // 32] >> (v % 32).int()) & 1
        off = (bits[st["mask_row"].long().clamp(min=0)] == 0) & (st["mask_row"] >= 0)[:, None]
        x = x.masked_fill(off, -math.inf)
    top = x.amax(1, keepdim=True)
    at = torch.where(x == top, torch.arange(V, device="cuda"), V).amin(1)
    pick = torch.where(top[:, 0] > -math.inf, at, -1).int()
    ref = top.masked_fill(top == -math.inf, 0.0)
    return {"logits": x.to(st["logits"].dtype), "pick": pick, "lse": ref[:, 0] + (x - ref).exp().sum(1).log()}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    k = case["kind"]
    if k == "logits":
        rows, lse = [], []
        for b in range(case["B"]):
            x = st["logits"][b].double()
            past = st["hist"][b, :int(st["hist_len"][b])].long()
            n = torch.bincount(past, minlength=case["V"]).double()
            rep = st["rep"][b].double()
            x = torch.where(n > 0, x * torch.where(x > 0, 1 / rep, rep), x) - n * st["freq"][b].double() - (n > 0) * st["pres"][b].double()
            if case["bias"]:
                x.index_add_(0, st["bias_ids"][b].long(), st["bias"][b].double())
            x /= st["temp"][b].double()
            if case["masks"] and int(st["mask_row"][b]) >= 0:
                words = st["mask"][int(st["mask_row"][b])]
                bits = torch.stack([(words >> i) & 1 for i in range(32)], dim=1).reshape(-1)[:case["V"]]
                x[bits == 0] = -math.inf
            rows.append(x)
            lse.append(torch.logsumexp(x, 0))
        return {"logits": torch.stack(rows), "pick": None, "lse": torch.stack(lse)}
    B, h, h_kv, kq, kv = (case[n] for n in ("B", "h", "h_kv", "kq", "kv"))
    lens = st["lens"].tolist()
    if k == "evict":
        k_out, v_out, w_out = st["k_out"].double(), st["v_out"].double(), st["w_out"].double()
        for b in range(B):
            n, keep = lens[b], min(lens[b], case["keep"])
            old = max(n - case["recent"], 0)
            for g in range(h_kv):
                rank = torch.argsort(-st["w"][b, g, :old].double(), stable=True)[:keep - (n - old)]
                kept = torch.cat((rank.sort().values, torch.arange(old, n, device="cuda")))[-keep:] if n > keep else torch.arange(n, device="cuda")
                k_out[b, g, :keep], v_out[b, g, :keep], w_out[b, g, :keep] = st["k"][b, g, kept].double(), st["v"][b, g, kept].double(), st["w"][b, g, kept].double()
        return {"k_out": k_out, "v_out": v_out, "w_out": w_out, "lens_out": None, "idx": None}
    L = case["L"]
    if k == "append":
        rows = st["qkv"].double().view(B, L, -1)
        q, key, val = rows[..., :h * kq], rows[..., h * kq:(h + h_kv) * kq], rows[..., (h + h_kv) * kq:]
        out = {"k": st["k"].double(), "v": st["v"].double(), "w": st["w"].double()}
        q, key, val = q.reshape(B, L, h, kq), key.reshape(B, L, h_kv, kq), val.reshape(B, L, h_kv, kv)
        turned = torch.empty_like(q)
        for b in range(B):
            kb = key[b]
            if case["rope"]:
                p = int(st["pos"][b])
                z = torch.complex(st["cos"][:, p:p + L].double(), st["sin"][:, p:p + L].double()).transpose(0, 1)      # [L, h_kv, kq / 2]
                kb = torch.view_as_real(torch.view_as_complex(kb.reshape(L, h_kv, -1, 2)) * z).reshape(L, h_kv, kq)
                zq = z[:, torch.arange(h, device="cuda") // (h // h_kv)]
                turned[b] = torch.view_as_real(torch.view_as_complex(q[b].reshape(L, h, -1, 2)) * zq).reshape(L, h, kq)
            s = lens[b] - L
            out["k"][b, :, s:s + L], out["v"][b, :, s:s + L], out["w"][b, :, s:s + L] = kb.transpose(0, 1), val[b].transpose(0, 1), 0.0
        return {**out, **({"q": turned.reshape(B * L, h * kq)} if case["rope"] else {})}
    P, scale = case["P"], _scale(case)
    if 2 * h * (kq + kv) * B * L * (P + case["own"]) > 4e12:
        return None
    o = torch.zeros(B, L, h, kv, device="cuda", dtype=torch.float64)
    lse = torch.zeros(B, h, L, device="cuda", dtype=torch.float64)
    w = st["w"].double() if case["weights"] else None
    q, pk, pv = st["q"].double().view(B, L, h, kq), st["pk"].double(), st["pv"].double()
    for b in range(B):
        n = lens[b]
        for g in range(h_kv):
            heads = slice(g * (h // h_kv), (g + 1) * (h // h_kv))
            keys, vals = torch.cat((pk[g], st["k"][b, g, :n].double())), torch.cat((pv[g], st["v"][b, g, :n].double()))
            s = q[b, :, heads].transpose(0, 1).reshape(-1, kq).mul(scale) @ keys.T                  # [group * L, P + n]
            late = torch.arange(P + n, device="cuda") >= P + n - L + 1 + torch.arange(L, device="cuda")[:, None]
            s = s.view(-1, L, P + n).masked_fill(late, -math.inf)
            z = torch.logsumexp(s, -1, keepdim=True)
            p = torch.exp(s - z.masked_fill(z == -math.inf, 0.0))
            lse[b, heads] = z[..., 0]
            o[b, :, heads] = (p @ vals).transpose(0, 1)
            if w is not None:
                w[b, g, :n] += p[..., P:].sum((0, 1))
    return {"o": o.reshape(B * L, h * kv), "lse": lse, **({"w": w} if w is not None else {})}
