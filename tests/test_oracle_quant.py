"""The oracle of serving in eight bits against values worked out by hand and against torch's own 8-bit type."""
import numpy as np
import torch

from oracle import quant_oracle as Q


def test_rows():
    q, s = Q.quant_rows(np.array([[1.0, -2.0, 127.0, 0.5, 1.5, 2.5], [0, 0, 0, 0, 0, 0], [np.inf, 1, 1, 1, 1, 1]], np.float32))
    assert q.tolist() == [[1, -2, 127, 0, 2, 2], [0] * 6, [0] * 6] and s[0] == 1.0 and s[1] == 0.0 and np.isnan(s[2])


def test_products():
    y, off = Q.contract_quant(np.array([[1, 2]], np.int8), [0.5], np.array([[3, 4], [-1, 1]], np.int8), [2.0, 1.0], bias=[1.0, 0.0])
    assert y.tolist() == [[12.0, 0.5]] and (off > 0).all()
    y, _ = Q.contract_quant(np.array([[1, 2]], np.int8), [1.0], np.array([[1, 0], [0, 1]], np.int8), [1.0, 1.0], act=Q.ACT_SWIGLU)
    assert np.allclose(y, [[2.0 / (1.0 + np.exp(-1.0))]])


def test_the_8_bit_type():
    x = np.concatenate([np.linspace(-448, 448, 4001), np.linspace(-0.05, 0.05, 4001), 2.0 ** np.arange(-12, 9)])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(Q.e4m3(x.astype(np.float32)), want)
    assert np.isnan(Q.e4m3(np.inf)) and np.isnan(Q.e4m3(np.nan))


def test_scales():
    for top, want in ((448.0, 1.0), (448.5, 2.0), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7), (0.0, 2.0 ** -100), (3.3e38, 2.0 ** 120)):
        assert Q.block_scale([0.0, -top, np.nan]) == want


def test_append_brings_earlier_rows_along():
    cache = {"k": np.zeros((1, 1, 4, 2)), "v": np.zeros((1, 1, 4, 2)), "k_scale": np.ones((1, 1, 1)), "v_scale": np.ones((1, 1, 1))}
    cache["k"][0, 0, 0] = [448.0, 2.0 ** -6]
    _, out = Q.append(np.array([[0, 0, 896.0, 1.0, 1.0, 2.0]]), cache, [2], 1, 4)
    assert out["k_scale"][0, 0, 0] == 2.0 and out["k"][0, 0, 0].tolist() == [224.0, 2.0 ** -7] and out["k"][0, 0, 1].tolist() == [448.0, 0.5]
    assert out["v_scale"][0, 0, 0] == 1.0 and out["v"][0, 0, 1].tolist() == [1.0, 2.0]


def test_attention_joins_other_keys():
    cache = {"k": np.zeros((1, 1, 2, 2)), "v": np.array([[[[1.0, 2.0], [3.0, 4.0]]]]), "k_scale": np.ones((1, 1, 1)), "v_scale": np.full((1, 1, 1), 2.0)}
    r = Q.attn(np.ones((1, 2)), cache, [2], 1, 1.0, 16, o_in=np.array([[10.0, 10.0]]), lse_in=np.full((1, 1, 1), np.log(2.0)))
    assert np.allclose(r["o"], [[(2 + 6 + 20) / 4, (4 + 8 + 20) / 4]]) and np.allclose(r["lse"], np.log(4.0))


def test_tokens():
    x = np.log([0.5, 0.3, 0.15, 0.05])
    assert [Q.sample(x, u)[0] for u in (0.0, 0.49, 0.51, 0.81, 0.96)] == [0, 0, 1, 2, 3]
    assert Q.sample(x, 0.99, top_k=2)[0] == 1 and Q.sample(x, 0.99, top_p=0.79)[0] == 1 and Q.sample(x, 0.99, top_p=0.81)[0] == 2
    assert Q.sample(x, 0.99, min_p=0.35)[0] == 1 and abs(Q.sample(x, 0.1, top_k=2)[1] - 0.625) < 1e-12
    assert Q.sample(x, 0.99, temperature=0.0) == (0, 1.0, 1.0) and Q.sample([-np.inf, np.nan], 0.5)[:2] == (-1, 0.0)
    assert Q.sample([1.0, np.inf, 2.0, np.inf], 0.6)[:2] == (3, 0.5) and Q.sample([2.0, 2.0, 2.0], 0.99, top_k=2)[0] == 1
