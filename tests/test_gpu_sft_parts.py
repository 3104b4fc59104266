"""pipeline.SFTStep on a batch in several parts: their gradients added up are the whole batch's, and a table's gradient of all parts is not
clipped beside a weight's of the last."""
import numpy as np
import pytest
import torch

from oracle import sft_oracle as O
from parity import npy

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


def f64(t):
    return t.detach().double().cpu().numpy()


def setup(N, K, V, columns=False):
    g = torch.Generator().manual_seed(5)
    E, W = torch.randn(V, K, generator=g).to(BF16).cuda(), (torch.randn(K, V, generator=g) / K ** 0.5).to(BF16).cuda()
    tokens = torch.randint(0, V, (N,), generator=g, dtype=I32)
    labels = tokens.roll(-1)
    labels[::9] = -100
    mask = (torch.rand(N, generator=g) > 0.2).to(torch.uint8)
    return E, W.t().contiguous().t() if columns else W, tokens.cuda(), labels.cuda(), mask.cuda()


@pytest.mark.parametrize("columns", [False, True])
def test_parts_add_up_to_the_batch(P, columns):
    from paper_2403_17031_b200.pipeline import SFTStep
    N, K, V, parts = 600, 64, 1008, 3
    E, W, tokens, labels, mask = setup(N, K, V, columns)
    n = N // parts
    denom = ((mask != 0) & (labels != -100)).sum().float().reshape(1)
    step = SFTStep(W, n, padding_id=1, grad_dtype=F32)
    dW, loss = torch.zeros((K, V) if not columns else (V, K), device="cuda"), 0.0
    for i in range(parts):
        at = slice(i * n, (i + 1) * n)
        h = step.embed(E, tokens[at])
        o = step.loss(h, W, labels[at], mask[at], denom=denom)
        step.grad_embed(o["dH"], tokens[at], accumulate=i > 0)
        dW += o["dW"].t() if columns else o["dW"]
        loss += float(o["loss"])
    real = (npy(mask) != 0) & (npy(labels) != -100)
    want = O.xent(f64(E[tokens.long()]), f64(W), npy(labels), real, 1.0)
    dE, _ = O.embed_bwd(want["dH"], npy(tokens), V, 1.0, 1)
    total = dW.t() if columns else dW
    # norms of rounding errors, each far below its worst case in all elements at once: half a step of 2^-8 of U, of a H or dH, of a part's result
    near = lambda a, b: np.linalg.norm(f64(a) - b) <= 2.0 ** -8 * np.linalg.norm(b)      # noqa: E731
    assert abs(loss - want["loss"]) < 1e-4 and near(total, want["dW"]) and near(step.out["dE"], dE)
    before = [total.clone(), step.out["dE"].clone()]
    with pytest.raises(ValueError):
        step.clip(0.01)
    assert torch.equal(step.out["dE"], before[1])
    norm = step.clip(0.01, dW=total)
    clipped, size, c = O.grad_clip([f64(t) for t in before], 0.01, 1.0)
    assert c < 1 and abs(float(norm[0]) - size) < 1e-6 * size and abs(float(norm[1]) - c) < 1e-6
    assert near(total, clipped[0]) and near(step.out["dE"], clipped[1])
    step.loss(step.embed(E, tokens[:n]), W, labels[:n], mask[:n])                        # the next batch, whole
    step.grad_embed(step.out["dH"], tokens[:n])
    step.clip(0.01)


def test_a_table_used_twice_in_a_part_and_a_frozen_one(P):
    """Two gradients on the same loss, a table's gradient cleared by the caller, and steps without one are no mixture."""
    from paper_2403_17031_b200.pipeline import SFTStep
    E, W, tokens, labels, mask = setup(100, 64, 304)
    step = SFTStep(W, 100)
    for _ in range(2):
        o = step.loss(step.embed(E, tokens), W, labels, mask)
        step.grad_embed(o["dH"], tokens)
        step.grad_embed(o["dH"], labels.clamp(min=0), accumulate=True)
        step.clip(1.0)
    for _ in range(2):
        o = step.loss(step.embed(E, tokens), W, labels, mask)
        o["dE"].zero_()
        step.grad_embed(o["dH"], tokens, accumulate=True)
        step.clip(1.0)
    o["dE"].zero_()
    for _ in range(2):
        step.loss(step.embed(E, tokens), W, labels, mask)
        step.clip(1.0)
    assert step.device_status() == 0


def test_a_clip_that_is_refused_changes_nothing(P):
    from paper_2403_17031_b200.pipeline import SFTStep
    E, W, tokens, labels, mask = setup(100, 64, 304)
    step = SFTStep(W, 100)
    for i in range(2):
        o = step.loss(step.embed(E, tokens), W, labels, mask)
        step.grad_embed(o["dH"], tokens, accumulate=i > 0)
    with pytest.raises(P.PPOError):
        step.clip(0.0, dW=o["dW"].clone())
    with pytest.raises(ValueError):
        step.clip(1.0)
    step.clip(1.0, dW=o["dW"].clone())
