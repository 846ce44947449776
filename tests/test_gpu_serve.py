"""The serving harness against the stack's own forward pass over the whole sequence: prefix, prompts and single tokens give the logits that the
full forward gives at the same position; evictions, masks and penalties run through it as a program would use them."""
import numpy as np
import pytest
import torch

from paper_2511_11641_amd import binding as B
from paper_2511_11641_amd.serve import Server, main
from paper_2511_11641_amd.stack import DecoderStack
from util import host

pytestmark = pytest.mark.gpu
VOCAB = 512


@pytest.fixture(scope="module")
def ctx():
    return B.Context("cuda:0")


def _stack(ctx, gated, L, h_kv=4, d_h=32, keep=(1, 2), seed=3):
    cfg = dict(B=1, L=L, d=128, h=4, h_kv=h_kv, d_h=d_h, d_ff=256, gated=gated, rope=gated, bias=not gated)
    st = DecoderStack(ctx, cfg, 2, VOCAB, keep=keep, seed=seed, train=False)
    for ly in st.layers:                                 # weights whose attention and activations are worth comparing
        for blk in (ly.attn["w"], ly.ffn["w"]):
            for n in ("wqkv_c", "wo_c", "w1_c", "w2_c"):
                if hasattr(blk, n):
                    getattr(blk, n).mul_(5.0)
    return st


@pytest.mark.parametrize("gated,h_kv,d_h,keep", [(True, 4, 32, (1, 2)), (True, 2, 64, (3, 4)), (False, 4, 64, (1, 2)), (True, 1, 128, (1, 1))])
@pytest.mark.parametrize("P,prompt", [(70, 5), (200, 1)])
def test_logits_are_those_of_the_whole_sequence(ctx, gated, h_kv, d_h, keep, P, prompt):
    Bsz, steps = 3, 4
    total = P + prompt + steps - 1
    st = _stack(ctx, gated, total, h_kv, d_h, keep)
    g = torch.Generator(device="cuda").manual_seed(P)
    ids = torch.randint(0, VOCAB, (Bsz, total), device="cuda", generator=g)
    ids[:, :P] = ids[:1, :P]
    want = [host(st.forward(ids[b].contiguous())) for b in range(Bsz)]
    srv = Server(st, Bsz, 24, total)
    srv.set_prefix(ids[0, :P].contiguous())
    at = P
    for n in [prompt] + [1] * (steps - 1):
        got = host(srv.feed(ids[:, at:at + n].contiguous()))
        at += n
        for b in range(Bsz):
            err = np.linalg.norm(got[b] - want[b][at - 1]) / np.linalg.norm(want[b][at - 1])
            assert err < 2e-2, (b, at, err)
    assert srv.lens.tolist() == [at - P] * Bsz and srv.pos.tolist() == [at] * Bsz


def test_without_a_prefix_and_with_one_request(ctx):
    st = _stack(ctx, True, 20)
    ids = torch.randint(0, VOCAB, (1, 20), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    want = host(st.forward(ids[0].contiguous()))
    srv = Server(st, 1, 32, 32, evictable=False)
    srv._caches()
    got = host(srv.feed(ids[:, :19].contiguous()))
    assert np.linalg.norm(got[0] - want[18]) / np.linalg.norm(want[18]) < 2e-2
    got = host(srv.feed(ids[:, 19:].contiguous()))
    assert np.linalg.norm(got[0] - want[19]) / np.linalg.norm(want[19]) < 2e-2


def test_evicted_keys_are_those_with_the_least_attention(ctx):
    st = _stack(ctx, True, 8, h_kv=2)
    g = torch.Generator(device="cuda").manual_seed(2)
    prefix, ids = torch.randint(0, VOCAB, (40,), device="cuda", generator=g), torch.randint(0, VOCAB, (4, 30), device="cuda", generator=g)
    srv = Server(st, 4, 32, 100)
    srv.set_prefix(prefix)
    srv.feed(ids)
    old = [(ly["kv"][0].clone(), ly["w"].clone()) for ly in srv.layers]
    # every query gives its own keys and the prefix a weight of one; the own part is what is accumulated
    assert all((w.sum(2) > 0).all() and (w.sum(2) <= 2 * 30 + 1e-3).all() for _, w in old)
    srv.evict(30, 4)                                     # nothing to do: everything stays
    assert all(torch.equal(ly["kv"][0][:, :, :30], k[:, :, :30]) and torch.equal(ly["w"][:, :, :30], w[:, :, :30]) for ly, (k, w) in zip(srv.layers, old))
    srv.evict(12, 4)
    assert srv.lens.tolist() == [12] * 4 and srv.pos.tolist() == [70] * 4 and srv.longest == 12
    for ly, (k, w) in zip(srv.layers, old):
        order = w[:, :, :26].sort(dim=2, descending=True, stable=True).indices[:, :, :8].sort(dim=2).values
        rows = torch.cat((order, torch.arange(26, 30, device="cuda").expand(4, 2, 4)), dim=2)
        assert torch.equal(ly["kv"][0][:, :, :12], k.gather(2, rows[..., None].expand(-1, -1, -1, k.shape[3])))
        assert torch.equal(ly["w"][:, :, :12], w.gather(2, rows))
    logits = srv.feed(ids[:, :1].contiguous())           # and the next token goes behind them
    assert srv.lens.tolist() == [13] * 4 and torch.isfinite(logits).all()


def test_generate_with_controls(ctx):
    st = _stack(ctx, True, 8)
    g = torch.Generator(device="cuda").manual_seed(4)
    prefix, prompts = torch.randint(0, VOCAB, (33,), device="cuda", generator=g), torch.randint(0, VOCAB, (3, 6), device="cuda", generator=g)
    srv = Server(st, 3, 16, 100)
    srv.set_prefix(prefix)
    free = srv.generate(prompts, 30, keep=8, recent=2)
    srv.set_prefix(prefix)
    assert torch.equal(free, srv.generate(prompts, 30, keep=8, recent=2)), "not the same twice"
    allowed = torch.arange(0, VOCAB, 37)
    words = torch.zeros((1, VOCAB // 32), dtype=torch.int64)
    for v in allowed.tolist():
        words[0, v // 32] |= 1 << (v % 32)
    mask = torch.where(words >= 1 << 31, words - (1 << 32), words).int().cuda()
    srv.set_prefix(prefix)
    out = srv.generate(prompts, 10, keep=8, presence=torch.full((3,), 1000.0, device="cuda"), mask=mask, mask_row=torch.tensor([0, 0, -1], dtype=torch.int32, device="cuda"))
    assert set(out[:2].flatten().tolist()) <= set(allowed.tolist())
    for b in range(3):                                   # a presence penalty that large: no token twice, none of the prompt's
        row = out[b].tolist()
        assert len(set(row)) == len(row) and not set(row) & set(prompts[b].tolist())


def test_the_command_runs(ctx, capsys):
    main(["--layers", "1", "--batch", "4", "--prefix", "100", "--prompt", "7", "--steps", "12", "--cap", "12"])
    assert '"tokens_per_s"' in capsys.readouterr().out
