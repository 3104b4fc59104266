"""Pins of oracle/topk_oracle.py and oracle/fp8_oracle.py to closed forms, finite differences and library routines."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as F
from oracle import topk_oracle as K


def test_topk_uniform_and_two_token_rows():
    o = K.topk(np.zeros((1, 8)), np.array([[3]]), 8, 0.7)
    assert abs(o["lse"][0] - np.log(8)) < 1e-14 and abs(o["entropy"][0] - np.log(8)) < 1e-14
    assert o["top_ids"][0].tolist() == list(range(8))          # ties: lowest index first
    x = np.array([[0.0, np.log(3.0), -np.inf]])
    o = K.topk(x, np.array([[0, 1, 2]]), 3, 1.0)
    assert np.allclose(np.exp(o["logprob"][0]), [0.25, 0.75, 0.0]) and o["top_ids"][0].tolist() == [1, 0, 2]
    assert abs(o["entropy"][0] - (2 * np.log(2) - 0.75 * np.log(3))) < 1e-14


def test_topk_rows_without_a_distribution():
    x = np.array([[np.nan, 1, 2], [np.inf, 0, 0], [-np.inf] * 3, [-3e38] * 3, [1, 2, 3]])
    o = K.topk(x, np.zeros((5, 1), int), 2, 1.0, mask=[1, 1, 1, 1, 0])
    assert np.isnan(o["lse"][:4]).all() and (o["top_ids"] == -1).all() and o["lse"][4] == 0


def test_topk_against_the_library():
    x = np.random.default_rng(0).normal(size=(5, 33)) * 3
    o = K.topk(x, np.arange(5)[:, None], 7, 0.7)
    z = torch.from_numpy(x / 0.7)
    lp = torch.log_softmax(z, 1)
    assert np.allclose(o["lse"], torch.logsumexp(z, 1)) and np.allclose(o["entropy"], torch.distributions.Categorical(logits=z).entropy())
    v, i = torch.topk(lp, 7)
    assert np.array_equal(o["top_ids"], i.numpy()) and np.allclose(o["top_logprob"], v.numpy())
    assert np.allclose(o["logprob"][:, 0], lp[torch.arange(5), torch.arange(5)])


def test_topk_gradient_by_central_differences():
    rng = np.random.default_rng(1)
    x, tau = rng.normal(size=(2, 9)), 0.7
    ids = np.array([[1, 1, 4], [8, 0, 8]])                     # an index given twice
    g, dh, dl = rng.normal(size=(2, 3)), rng.normal(size=2), rng.normal(size=2)

    def value(y):
        o = K.topk(y, ids, 0, tau)
        return (o["logprob"] * g).sum() + (o["entropy"] * dh).sum() + (o["lse"] * dl).sum()
    o = K.topk(x, ids, 0, tau)
    d, size = K.topk_bwd(x, ids, g, o["lse"], tau, o["entropy"], dh, dl)
    for r in range(2):
        for j in range(9):
            e = np.zeros_like(x)
            e[r, j] = 1e-5
            assert abs((value(x + e) - value(x - e)) / 2e-5 - d[r, j]) < 1e-8
    assert (size >= np.abs(d) - 1e-12).all()


def test_e4m3_is_the_types_rounding():
    rng = np.random.default_rng(2)
    v = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.uniform(-5, 3, 4000), np.arange(-512, 512) / 1024.0, [447.9, 448, 464, 1e9]])
    v = v.astype(np.float32)
    want = torch.from_numpy(v).clamp(-448, 448).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(F.e4m3(v.astype(np.float64)), want)


@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_keeps_every_value_within_half_a_step(rows):
    x = (np.random.default_rng(3).normal(size=(200, 300)) * 5).astype(np.float32)
    q, s = F.quantize(x, rows)
    assert s.shape == ((3, 200) if rows == 1 else (2, 3)) and np.abs(q).max() == 448
    back = F.dequantize(q, s, rows)
    step = np.maximum(2.0 ** -4 * np.abs(x), F.dequantize(np.full_like(q, 2.0 ** -10), s, rows))
    assert (np.abs(back - x) <= step * (1 + 1e-6)).all()


def test_product_of_exact_operands():
    a = np.random.default_rng(4).integers(-4, 5, size=(3, 300)).astype(np.float64)
    b = np.random.default_rng(5).integers(-4, 5, size=(130, 300)).astype(np.float64)
    sa, sb = np.full((3, 3), 0.5), np.array([[1.0, 2.0, 4.0], [8.0, 1.0, 1.0]])
    c, size = F.matmul(a, sa, b, sb, 128)
    f = np.repeat(np.repeat(sb, 128, 0)[:130], 128, 1)[:, :300] * 0.5
    assert np.array_equal(c, a @ (b * f).T) and (size >= np.abs(c)).all()
