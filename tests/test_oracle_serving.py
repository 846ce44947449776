"""The serving oracle against values worked out by hand and against independent formulations (CPU)."""
import numpy as np
import torch

from oracle import serving_oracle as S


def test_attention_is_a_softmax_over_all_visible_keys():
    rng = np.random.default_rng(0)
    B, L, h, h_kv, e, f, P, cap = 3, 4, 6, 2, 8, 5, 7, 9
    q, k, v = rng.standard_normal((B * L, h * e)), rng.standard_normal((B, h_kv, cap, e)), rng.standard_normal((B, h_kv, cap, f))
    pk, pv, lens = rng.standard_normal((h_kv, P, e)), rng.standard_normal((h_kv, P, f)), [9, 4, 6]
    got = S.prefix_attn(q, k, v, lens, h, 0.3, pk, pv)
    for b in range(B):
        keys = torch.tensor(np.concatenate((pk, k[b, :, :lens[b]]), axis=1)).repeat_interleave(h // h_kv, 0)
        vals = torch.tensor(np.concatenate((pv, v[b, :, :lens[b]]), axis=1)).repeat_interleave(h // h_kv, 0)
        x = torch.tensor(q[b * L:(b + 1) * L]).view(L, h, e).transpose(0, 1)
        mask = torch.ones(L, P + lens[b], dtype=torch.bool).tril(diagonal=P + lens[b] - L)
        s = (x @ keys.transpose(1, 2) * 0.3).masked_fill(~mask, -torch.inf)
        p = s.softmax(-1)
        assert np.allclose(got["o"][b * L:(b + 1) * L], (p @ vals).transpose(0, 1).reshape(L, -1).numpy(), atol=1e-12)
        assert np.allclose(got["lse"][b], s.logsumexp(-1).numpy(), atol=1e-12)
        assert np.allclose(got["w"][b, :, :lens[b]], p[..., P:].reshape(h_kv, -1, L, lens[b]).sum((1, 2)).numpy(), atol=1e-12)


def test_queries_without_keys_have_no_weight():
    k, v = np.ones((1, 1, 4, 2)), np.ones((1, 1, 4, 2))
    got = S.prefix_attn(np.ones((3, 2)), k, v, [1], 1, 1.0)
    assert got["lse"][0, 0].tolist()[:2] == [-np.inf, -np.inf] and np.isfinite(got["lse"][0, 0, 2])
    assert got["o"].tolist() == [[0, 0], [0, 0], [1, 1]] and got["w"][0, 0].tolist() == [1, 0, 0, 0]


def test_evict_by_hand():
    w = np.array([[[0.5, 2.0, 0.5, np.nan, 0.5, 9.0, 0.0, 0.0]]])
    assert S.evict(w, [8], 5, 2) == ([[[0, 1, 5, 6, 7]]], [5])          # of three 0.5 the first
    assert S.evict(w, [8], 8, 2) == ([[list(range(8))]], [8])
    assert S.evict(w, [5], 2, 0) == ([[[0, 1]]], [2])
    assert S.evict(w, [8], 3, 3) == ([[[5, 6, 7]]], [3])
    assert S.evict(w, [4], 3, 0) == ([[[0, 1, 2]]], [3])                # NaN goes first


def test_turn_and_append():
    assert np.allclose(S.turn([1.0, 0.0, 0.0, 2.0], np.array([0.0, 1.0]), np.array([1.0, 0.0])), [0, 1, 0, 2])
    qkv = np.arange(2 * 6, dtype=float).reshape(2, 6)                    # one request, two tokens; h = h_kv = 1, e = f = 2
    q, k, v, w = S.append(qkv, np.zeros((1, 1, 3, 2)), np.zeros((1, 1, 3, 2)), [3], 1, w=np.ones((1, 1, 3)))
    assert q.tolist() == [[0, 1], [6, 7]] and k[0, 0].tolist() == [[0, 0], [2, 3], [8, 9]] and v[0, 0, 2].tolist() == [10, 11]
    assert w[0, 0].tolist() == [1, 0, 0]
    q, k, v, _ = S.append(qkv, np.zeros((1, 1, 3, 2)), np.zeros((1, 1, 3, 2)), [1], 1)       # the first token has no row
    assert q.tolist() == [[0, 0], [6, 7]] and k[0, 0, 0].tolist() == [8, 9]


def test_logits_by_hand():
    x, pick, lse = S.logits_process([[2.0, -2.0, 1.0, 4.0]], history=[[0, 1, 1, 9]], repetition=[2.0], frequency=[0.25], presence=[0.5],
                                    temperature=[0.5], bias_ids=[[2, 2, -1]], bias=[[1.0, 0.5, 7.0]], mask=[[0b0111]], mask_row=[0])
    assert x[0].tolist() == [0.5, -10.0, 5.0, -np.inf] and pick[0] == 2
    assert np.isclose(lse[0], np.log(np.exp(0.5) + np.exp(-10.0) + np.exp(5.0)))
    x, pick, lse = S.logits_process([[1.0, 1.0], [0.0, np.nan]], mask=[[0]], mask_row=[0, -1])
    assert pick.tolist() == [-1, 0] and lse[0] == -np.inf and np.isnan(lse[1])
