"""Pins of oracle/sft_oracle.py to closed forms, finite differences and library routines."""
import numpy as np
import pytest
import torch

from oracle import sft_oracle as O


def test_uniform_rows_and_a_hand_case():
    o = O.xent(np.zeros((3, 4)), np.ones((4, 8)), np.array([0, 5, 7]), [1, 1, 1], 0.7)
    assert np.allclose(o["nll"], np.log(8)) and np.isclose(o["loss"], np.log(8))
    assert np.allclose(o["D"][1], np.where(np.arange(8) == 5, 1 / 8 - 1, 1 / 8) / (3 * np.float32(0.7)))
    # logits (0, ln 3): p = (1/4, 3/4)
    o = O.xent(np.array([[1.0]]), np.array([[0.0, np.log(3.0)]]), np.array([0]), [1], 1.0, scale=2.0)
    assert np.isclose(o["loss"], np.log(4)) and np.allclose(o["D"], [[-1.5, 1.5]]) and np.allclose(o["dH"], 1.5 * np.log(3))


@pytest.mark.parametrize("denom", [None, 11.0])
def test_gradients_against_differences_and_the_library(denom):
    g = np.random.default_rng(3)
    H, W = g.normal(size=(5, 3)), g.normal(size=(3, 7))
    labels, real = g.integers(0, 7, 5), np.array([1, 0, 1, 1, 0])
    o = O.xent(H, W, labels, real, 1.0, denom=denom)
    f = lambda h, w: O.xent(h, w, labels, real, 1.0, denom=denom)["loss"]          # noqa: E731
    for x, d, at in ((H, o["dH"], 0), (W, o["dW"], 1)):
        for i in np.ndindex(x.shape):
            step = np.zeros_like(x)
            step[i] = 1e-5
            a, b = ((H + step, W), (H - step, W)) if at == 0 else ((H, W + step), (H, W - step))
            assert abs((f(*a) - f(*b)) / 2e-5 - d[i]) < 1e-9
    lab = torch.from_numpy(np.where(real, labels, -100))
    want = torch.nn.functional.cross_entropy(torch.from_numpy(H @ W), lab, reduction="sum") / (denom or 3)
    assert np.isclose(o["loss"], float(want), rtol=1e-13)
    assert not o["dH"][1].any() and o["nll"][4] == 0


def test_bad_label_and_empty_selection():
    H, W = np.ones((2, 3)), np.ones((3, 4))
    o = O.xent(H, W, np.array([0, 4]), [1, 1], 1.0)
    assert np.isnan(o["loss"]) and np.isnan(o["nll"][1]) and np.isfinite(o["nll"][0]) and np.isnan(o["dW"]).all()
    o = O.xent(H, W, np.array([0, 1]), [0, 0], 1.0)
    assert o["loss"] == 0 and not o["dW"].any() and not o["dH"].any()


def test_embedding_against_the_library():
    g = np.random.default_rng(4)
    table, tokens, dY = g.normal(size=(9, 5)), g.integers(0, 9, 40), g.normal(size=(40, 5))
    assert np.allclose(O.embed(table, tokens, 2.0), 2 * table[tokens])
    t = torch.from_numpy(table).requires_grad_(True)
    y = torch.nn.functional.embedding(torch.from_numpy(tokens), t, padding_idx=3) * 2.0
    d, size = O.embed_bwd(dY, tokens, 9, 2.0, padding_id=3)
    assert np.allclose(d, torch.autograd.grad(y, t, torch.from_numpy(dY))[0].numpy()) and not d[3].any()
    assert (size >= np.abs(d) - 1e-12).all()
    assert np.isnan(O.embed(table, np.array([9, -1]), 1.0)).all()


def test_grad_clip_closed_forms():
    out, norm, coef = O.grad_clip([np.array([3.0]), np.array([[4.0]])], 2.5, 1.0)
    assert norm == 5 and coef == 0.5 and out[0][0] == 1.5 and out[1][0, 0] == 2
    out, norm, coef = O.grad_clip([np.array([3.0, 4.0])], 10.0, -0.5)
    assert norm == 2.5 and coef == 1 and out[0].tolist() == [-1.5, -2.0]
    assert O.grad_clip([np.zeros(3)], 1.0, 1.0)[1:] == (0.0, 1.0)
