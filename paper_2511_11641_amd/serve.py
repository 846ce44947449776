"""Serving a compact decoder stack token by token: a batch of requests behind one shared prefix, each with a cache of its own.

A harness, as :mod:`.stack` is for training: every kernel of a step is the library's.  The prefix runs once, as one sequence, through the
blocks' forward pass; its keys and values are kept once for all requests.  A request's own tokens - its prompt, then one token a step -
go through the projection, into its cache (``ecospa_cache_append``: turned by the angles of the kept rotary blocks at its own position),
through the attention over prefix and cache (``ecospa_prefix_attn``), the output projection and the FFN block.  The last token's logits
are penalised, biased and masked (``ecospa_logits_process``), which also names the best token; by random numbers, one is drawn instead
(``ecospa_sample``).  When the caches are full, the keys that received the least attention leave (``ecospa_cache_evict``); positions go on
counting.

Two parts can be kept in 8 bits: the requests' own caches (``ecospa_quant_cache_append``, ``ecospa_quant_cache_attn``, joined with the
attention over the prefix, which stays bf16) and the weights that every step reads (``ecospa_quant_rows``, ``ecospa_contract_quant``).

``python -m paper_2511_11641_amd.serve`` runs a model of random weights this way and prints tokens per second.
"""
from __future__ import annotations

import argparse
import json
import time
from typing import Optional

import torch

from . import binding as B
from .stack import DecoderStack


class Server:
    """``Bsz`` requests on the compact weights of a :class:`.stack.DecoderStack` (its first estimate is done when it is built), with room
    for ``cap`` own tokens each and positions up to ``max_pos``.  Requests share no prefix until :meth:`set_prefix` gives them one.
    evictable: keep the attention weight of every own key (what :meth:`evict` goes by).  The stack's weights stay as they are while this
    object is in use: a new estimate needs a new one.
    cache_block: own caches in 8-bit floats with a scale for this many rows (16, 32, 64 or 128); these keep no attention weights, so
    evictable has to be False.  quant_weights: a copy of the weights in 8-bit integers, made here, is what :meth:`feed` multiplies by (the prefix,
    which runs once, goes through the stack's own)."""

    def __init__(self, stack: DecoderStack, Bsz: int, cap: int, max_pos: int, evictable: bool = True, cache_block: Optional[int] = None,
                 quant_weights: bool = False):
        if cache_block is not None and evictable:
            raise ValueError("caches in 8 bits keep no attention weights: evictable=False")
        self.st, self.ctx, self.B, self.cap, self.max_pos = stack, stack.ctx, Bsz, cap, max_pos
        assert stack.pos is None or max_pos <= stack.pos.w.shape[0], "positions beyond the learned table"
        bf, dev = torch.bfloat16, "cuda"
        self.P, self.longest = 0, 0               # tokens of the prefix; upper bound on the own lengths (known here, so that calls can be cut)
        self.used = 0                             # positions that every request has behind it, prefix and evicted tokens among them
        self.lens, self._no_lens = torch.zeros(Bsz, dtype=torch.int32, device=dev), torch.zeros(Bsz, dtype=torch.int32, device=dev)
        self.pos = torch.zeros(Bsz, dtype=torch.int32, device=dev)         # position of a request's next token
        self.layers, self.spare, self.block = [], None, cache_block
        quant = (lambda w: self.ctx.ecospa_quant_rows(w)) if quant_weights else lambda w: None
        for ly in stack.layers:
            a = ly.attn["w"]
            one = bf if cache_block is None else torch.float8_e4m3fn
            kv = lambda n: (torch.zeros((n, a.h_kv, cap, a.kp_qk), dtype=one, device=dev), torch.zeros((n, a.h_kv, cap, a.kp_vo), dtype=one, device=dev))
            self.layers.append({"attn": a, "ffn": ly.ffn["w"], "norm": ly.norm, "rope": a._rope_table(max_pos) if a.rope else None, "kv": kv(Bsz),
                                "w": torch.zeros((Bsz, a.h_kv, cap), dtype=torch.float32, device=dev) if evictable else None, "prefix": (None, None)})
            f = ly.ffn["w"]
            self.layers[-1]["quant"] = {n: quant(w) for n, w in (("wqkv", a.wqkv_c), ("wo", a.wo_c), ("w1", f.w1_c), ("w2", f.w2_c))}
            if cache_block is not None:
                self.layers[-1]["scales"] = [torch.zeros((Bsz, a.h_kv, -(-cap // cache_block)), dtype=torch.float32, device=dev) for _ in range(2)]
                self.layers[-1]["none"] = [torch.zeros((Bsz, a.h_kv, 1, n), dtype=bf, device=dev) for n in (a.kp_qk, a.kp_vo)]      # the cache of a prefix's attention
            if evictable and self.spare is None:  # what an eviction writes into; the cache it leaves is the next layer's
                self.spare = (*kv(Bsz), torch.zeros((Bsz, a.h_kv, cap), dtype=torch.float32, device=dev))
        self.lm_quant = quant(stack.lm.w)
        self._buffers, self._descs, self._codes = {}, {}, {}
        self._caches()                            # without a prefix until there is one

    def _buf(self, name: str, rows: int, width: int, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        key = (name, rows, width, dtype)
        if key not in self._buffers:
            self._buffers[key] = torch.empty((rows, width), dtype=dtype, device="cuda")
        return self._buffers[key]

    def _caches(self):
        for ly in self.layers:
            a, own_max, scale = ly["attn"], min(self.longest, self.cap), float(ly["attn"].d_h) ** -0.5
            if self.block is not None:
                ly["cache"] = B.QuantCache(*ly["kv"], *ly["scales"], self.lens, a.h, scale, self.block, own_max=own_max)
                ly["shared"] = B.KvCache(*ly["none"], self._no_lens, a.h, scale, *ly["prefix"], own_max=0) if self.P else None
                continue
            ly["cache"] = B.KvCache(*ly["kv"], self.lens, a.h, scale, *ly["prefix"], own_max=own_max)

    def _norm(self, ps, x, res, out, y):
        rms = self.st.rms
        self.ctx.ecospa_norm_fwd(B.NORM_RMS if rms else B.NORM_LAYER, x, ps[0].w, None if rms else ps[1].w, self.st.eps, y, res=res, x_out=out)
        return x if res is None else out

    def _embed(self, ids: torch.Tensor, first: torch.Tensor, L: int):
        """(token rows, position rows or None) of ids [Bsz * L], request b's at positions first[b] on."""
        st, T = self.st, ids.numel()
        x = self.ctx.ecospa_embed_fwd(ids, st.emb.w, self._buf("x", T, st.d))
        if st.pos is None:
            return x, None
        at = (first.view(-1, 1) + torch.arange(L, device="cuda")).reshape(-1).long()
        return x, self.ctx.ecospa_embed_fwd(at, st.pos.w, self._buf("at", T, st.d))

    def _mul(self, x, w, quant, bias, out, act: Optional[int] = None):
        """act(x w^T + bias), by the 8-bit copy of w where there is one (act: there alone)."""
        if quant is None:
            return self.ctx.ecospa_contract(x, False, w, False, bias=bias, out=out)
        codes = self._codes.get(x.shape)
        if codes is None:
            codes = self._codes[x.shape] = (torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(x.shape[0], dtype=torch.float32, device="cuda"))
        q, s = self.ctx.ecospa_quant_rows(x, *codes)
        return self.ctx.ecospa_contract_quant(q, s, *quant, bias=bias, act=act, out=out)

    def _ffn(self, f, x, quant=None):
        T = x.shape[0]
        if quant is not None and quant["w1"] is not None:
            mid = self._mul(x, None, quant["w1"], f.b1_c, self._buf("mid", T, f.kp), act=f.act)
            return self._mul(mid, None, quant["w2"], f.b2, self._buf("y", T, self.st.d))
        if (id(f), T) not in self._descs:         # descriptors of this object's own layers
            self._descs[id(f), T] = f.desc(T, 1)
        return self.ctx.ecospa_coupled_fwd(self._descs[id(f), T], x, self._buf("y", T, self.st.d), None)

    @torch.no_grad()
    def set_prefix(self, ids: torch.Tensor):
        """The prefix that every request starts with (int64 [P]; P <= max_pos): runs it once and empties the requests' own caches."""
        st, ctx, P = self.st, self.ctx, ids.numel()
        assert P <= self.max_pos, f"a prefix of {P} tokens, tables of {self.max_pos} positions"
        self.P, self.longest, self.used = P, 0, P
        self.lens.zero_()
        self.pos.fill_(P)
        one, whole = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((1,), P, dtype=torch.int32, device="cuda")
        x, res = self._embed(ids, one, P)
        x2, y = self._buf("x2", P, st.d), self._buf("h", P, st.d)
        for ly in self.layers:
            a = ly["attn"]
            x = self._norm(ly["norm"][0], x, res, x2, y)
            qkv = self._buf("qkv", P, a.wqkv_c.shape[0])
            saved = B.Saved(qkv.data_ptr(), self._buf("o", P, a.h * a.kp_vo).data_ptr(), B._ptr(self._lse(a.h * P)), None, None)
            d = B.BlockDesc.from_buffer_copy(a._desc)
            d.B, d.L = 1, P
            if a.rope:
                cos, sin = a._rope_table(P)
                d.rope_cos, d.rope_sin = cos.data_ptr(), sin.data_ptr()
            res = ctx.ecospa_coupled_fwd(d, y, self._buf("r", P, st.d), saved)
            # its keys (turned already) and values, a head's rows side by side
            pk = torch.empty((1, a.h_kv, P, a.kp_qk), dtype=torch.bfloat16, device="cuda")
            pv = torch.empty((1, a.h_kv, P, a.kp_vo), dtype=torch.bfloat16, device="cuda")
            ctx.ecospa_cache_append(B.KvCache(pk, pv, whole, a.h, 1.0), qkv)
            ly["prefix"] = (pk[0], pv[0])
            x = self._norm(ly["norm"][1], x, res, x2, y)
            res = self._ffn(ly["ffn"], y)
        self._caches()

    def _room(self, L: int):
        assert self.used + L <= self.max_pos, f"{L} tokens behind {self.used}, tables of {self.max_pos} positions"

    def _lse(self, n: int) -> torch.Tensor:
        if getattr(self, "_lse_buf", None) is None or self._lse_buf.numel() < n:
            self._lse_buf = torch.empty(n, dtype=torch.float32, device="cuda")
        return self._lse_buf

    @torch.no_grad()
    def feed(self, ids: torch.Tensor) -> torch.Tensor:
        """The next L tokens of every request (int64 [Bsz, L]) -> logits of the last ones, bf16 [Bsz, vocab] (a buffer of this object).
        Evictions make room in the caches, not in the tables: positions end with max_pos."""
        st, ctx = self.st, self.ctx
        n, L = ids.shape
        assert n == self.B, f"tokens of {n} requests, built for {self.B}"
        self._room(L)
        assert self.longest + L <= self.cap, "the caches are full: evict() first"
        T = self.B * L
        self.used += L
        self.longest += L
        self.lens += L
        x, res = self._embed(ids.reshape(-1), self.pos, L)
        x2, y = self._buf("x2", T, st.d), self._buf("h", T, st.d)
        for ly in self.layers:
            a, cache = ly["attn"], ly["cache"]
            cache.own_max = self.longest
            x = self._norm(ly["norm"][0], x, res, x2, y)
            w8 = ly["quant"]
            qkv = self._mul(y, a.wqkv_c, w8["wqkv"], a.bqkv_c, self._buf("qkv", T, a.wqkv_c.shape[0]))
            q, o = self._buf("q", T, cache.nq) if a.rope else qkv, self._buf("o", T, cache.no)
            if self.block is None:
                ctx.ecospa_cache_append(cache, qkv, self.pos, rope=ly["rope"], q=q if a.rope else None, weights=ly["w"])
                ctx.ecospa_prefix_attn(cache, q, o, weights=ly["w"], weights_out=ly["w"])
            else:
                ctx.ecospa_quant_cache_append(cache, qkv, self.pos, rope=ly["rope"], q=q if a.rope else None)
                front = (None, None)
                if ly["shared"] is not None:
                    front = (o, self._lse(T * a.h)[:T * a.h])
                    ctx.ecospa_prefix_attn(ly["shared"], q, *front)
                ctx.ecospa_quant_cache_attn(cache, q, o, o_in=front[0], lse_in=front[1])
            res = self._mul(o, a.wo_c, w8["wo"], a.bo, self._buf("r", T, st.d))
            x = self._norm(ly["norm"][1], x, res, x2, y)
            res = self._ffn(ly["ffn"], y, w8)
        self._norm(st.norm_f, x, res, x2, y)
        self.pos += L
        last = y.view(self.B, L * st.d)[:, (L - 1) * st.d:]
        return self._mul(last, st.lm.w, self.lm_quant, None, self._buf("logits", self.B, st.vocab))

    @torch.no_grad()
    def evict(self, keep: int, recent: int):
        """Cuts every cache down to `keep` keys per head: the last `recent` and those that received the most attention."""
        assert self.spare is not None, "built without the attention weights"
        new = torch.empty_like(self.lens)
        for ly in self.layers:
            k, v, w = self.spare
            self.ctx.ecospa_cache_evict(ly["cache"], ly["w"], keep, recent, k, v, new, w)
            self.spare = (*ly["kv"], ly["w"])
            ly["kv"], ly["w"] = (k, v), w
        self.lens.copy_(new)
        self.longest = min(self.longest, keep)
        self._caches()

    @torch.no_grad()
    def generate(self, prompts: torch.Tensor, steps: int, *, keep: Optional[int] = None, recent: int = 0, u: Optional[torch.Tensor] = None,
                 top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None, **control):
        """`steps` tokens behind the prompts (int64 [Bsz, L]), the best one each time after `control` (the keyword arguments of
        ``Context.ecospa_logits_process``: repetition, frequency, presence, temperature, bias_ids, bias, mask, mask_row); the
        history of the penalties is the prompt and what came since.  Full caches are cut down to `keep` keys.  -> int32 [Bsz, steps]; -1
        where no token was left to pick (everything masked, or not a number), and token 0 is fed in its place.
        u (float32 [steps, Bsz], in [0, 1)): tokens are drawn by these numbers instead, from what top_k (int32), top_p and min_p (each [Bsz] or None) leave;
        all of them on the GPU."""
        if u is None and not (top_k is None and top_p is None and min_p is None):
            raise ValueError("top_k, top_p and min_p restrict a draw: give its random numbers u")
        Bsz, L = prompts.shape
        if u is not None:
            if u.shape != (steps, Bsz) or u.dtype != torch.float32:
                raise ValueError(f"expected random numbers float32 [{steps}, {Bsz}], got {u.dtype} {tuple(u.shape)}")
            u, T = u.contiguous(), control.pop("temperature", None)      # the draw's own: its weights come from unrounded logits
            if not all(t is None or t.is_cuda for t in (u, T, top_k, top_p, min_p)):
                raise ValueError("random numbers and what restricts a draw have to be on the GPU")
            wide = self._buf("wide", Bsz, B.round_up(self.st.vocab, 8), torch.float32)[:, :self.st.vocab]
        self._room(L + max(steps - 1, 0))         # the last token is not fed
        history = torch.zeros((Bsz, L + steps), dtype=torch.int32, device="cuda")
        history[:, :L] = prompts
        seen = torch.full((Bsz,), L, dtype=torch.int32, device="cuda")
        logits = self.feed(prompts)
        for i in range(steps):
            pick, _ = self.ctx.ecospa_logits_process(logits, out=logits if u is None else wide, history=history, history_len=seen, **control)
            if u is not None:
                pick = self.ctx.ecospa_sample(wide, u[i], temperature=T, top_k=top_k, top_p=top_p, min_p=min_p)
            history[:, L + i] = pick
            if i + 1 == steps:
                break
            seen += 1
            if self.longest + 1 > self.cap:
                assert keep is not None, "the caches are full and no `keep` is given"
                self.evict(keep, recent)
            logits = self.feed(pick.clamp(min=0).long().view(-1, 1))
        return history[:, L:]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--prefix", type=int, default=4096)
    ap.add_argument("--prompt", type=int, default=61)
    ap.add_argument("--steps", type=int, default=128)
    ap.add_argument("--cap", type=int, default=160, help="own tokens a cache holds before it is cut down to half")
    ap.add_argument("--cache-block", type=int, choices=(16, 32, 64, 128), help="own caches in 8-bit floats, a scale for this many rows; all own tokens are kept")
    ap.add_argument("--quant-weights", action="store_true", help="weights in 8-bit integers")
    ap.add_argument("--top-p", type=float, help="draw tokens from this share of the probability instead of taking the best")
    ap.add_argument("--temperature", type=float, help="of the draw (1)")
    a = ap.parse_args(argv)
    if a.temperature is not None and a.top_p is None:
        ap.error("--temperature is that of a draw: give --top-p (1 draws from all tokens)")
    from .synth import CONFIGS
    cfg = dict(CONFIGS["c3_llama1b_layer"], B=1, L=64)
    st = DecoderStack(B.Context("cuda:0"), cfg, a.layers, 32000, keep=(1, 2), train=False)
    if a.cache_block:
        a.cap = a.prompt + a.steps
    srv = Server(st, a.batch, a.cap, a.prefix + a.prompt + a.steps, evictable=not a.cache_block, cache_block=a.cache_block, quant_weights=a.quant_weights)
    gen = torch.Generator(device="cuda").manual_seed(0)
    ids = lambda *s: torch.randint(0, 32000, s, device="cuda", generator=gen)
    prefix, prompts = ids(a.prefix), ids(a.batch, a.prompt)
    half = torch.full((a.batch,), 1.2, device="cuda")
    draw = {}
    if a.top_p is not None:
        each = lambda x: torch.full((a.batch,), x, device="cuda")
        draw = dict(u=torch.rand((a.steps, a.batch), device="cuda", generator=gen), top_p=each(a.top_p), temperature=each(1.0 if a.temperature is None else a.temperature))
    for timed in (False, True):
        srv.set_prefix(prefix)
        torch.cuda.synchronize()
        t = time.perf_counter()
        srv.generate(prompts, a.steps, keep=a.cap // 2, recent=a.cap // 8, repetition=half, **draw)
        torch.cuda.synchronize()
        t = time.perf_counter() - t
    print(json.dumps({"model": f"{a.layers} x c3_llama1b_layer, half-kept, random weights", "batch": a.batch, "prefix": a.prefix, "prompt": a.prompt,
                      "steps": a.steps, "cap": a.cap, "cache": f"e4m3, a scale for {a.cache_block} rows" if a.cache_block else "bf16", "weights": "int8" if a.quant_weights else "bf16",
                      "pick": "best" if a.top_p is None else f"drawn, top-p {a.top_p}", "tokens_per_s": round(a.batch * a.steps / t, 1), "ms_per_step": round(1e3 * t / a.steps, 4)}))


if __name__ == "__main__":
    main()
