"""pipeline.SFTStep: embedding, a small model, cross entropy, both gradients and clipping as a training step uses them, stage by stage against
the fp64 definitions (each stage given the library's own inputs to it), and the gradients of the whole against differences."""
import numpy as np
import pytest
import torch

from oracle import sft_oracle as O
from parity import npy

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


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


def setup(N, K, V, columns, seed=0):
    g = torch.Generator().manual_seed(seed)
    E = torch.randn(V, K, generator=g).to(BF16).cuda()
    W = (torch.randn(K, V, generator=g) / K ** 0.5).to(BF16).cuda()
    W = W.t().contiguous().t() if columns else W
    mid = (torch.randn(K, K, generator=g) / K ** 0.5).to(BF16).cuda()
    tokens = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    tokens[::6] = 1
    labels = tokens.roll(-1)
    labels[::9] = -100
    mask = torch.rand(N, generator=g) > 0.2
    return E, W, mid, tokens.cuda(), labels.cuda(), mask.to(torch.uint8).cuda()


def model(x, mid):
    """The caller's part: hidden states, and the way back."""
    h = (x.float() @ mid.float()).to(BF16)
    return h, lambda dh: (dh.float() @ mid.float().t()).to(BF16), lambda dh: x.float().t() @ dh.float()


@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("N,K,V,dtype", [(40, 64, 304, BF16), (700, 128, 1008, F32), (1500, 72, 2000, BF16)])
def test_a_step(P, N, K, V, dtype, columns):
    from paper_2403_17031_b200.pipeline import SFTStep
    E, W, mid, tokens, labels, mask = setup(N, K, V, columns)
    step = SFTStep(W, N, padding_id=1, embed_scale=2.0, grad_dtype=dtype, piece_rows=512)
    x = step.embed(E, tokens)
    h, back, weight = model(x, mid)
    o = step.loss(h, W, labels, mask)
    dmid = weight(o["dH"])
    step.grad_embed(back(o["dH"]), tokens)
    before = [o["dW"].clone(), o["dE"].clone(), dmid.clone()]
    norm = step.clip(0.01, [dmid]).clone()
    assert step.device_status() == 0
    assert np.array_equal(f64(x), O.embed(f64(E), npy(tokens), 2.0))                # doubling is exact
    want = O.xent(f64(h), f64(W), npy(labels), npy(mask) * (npy(labels) != -100), 1.0)
    # norms of rounding errors: U and a H half a step of 2^-8, the result another; each is far below its worst case in all elements at once
    near = lambda a, b: np.linalg.norm(f64(a) - b) <= 2.0 ** -8 * np.linalg.norm(b)      # noqa: E731
    assert abs(float(o["loss"]) - want["loss"]) < 1e-4 and near(o["dH"], want["dH"]) and near(before[0], want["dW"])
    dE, _ = O.embed_bwd(f64(back(o["dH"])), npy(tokens), V, 2.0, 1)
    assert near(before[1], dE) and not before[1][1].any()
    clipped, n, c = O.grad_clip([f64(t) for t in before], 0.01, 1.0)
    assert abs(float(norm[0]) - n) < 1e-6 * n and abs(float(norm[1]) - c) < 1e-6 and c < 1
    assert near(o["dW"], clipped[0]) and near(o["dE"], clipped[1]) and near(dmid, clipped[2])


def test_gradients_of_the_whole_against_differences(P):
    """The loss moves along the gradients as they say. Along a direction d of length t the loss changes by t (g . d) + O(t^2); a central
    difference is off by O(t^2) of that, by the rounding of the weights moved (half a step of bf16 each, in both copies, which is why the
    direction taken is the one between the rounded copies) and by the losses' own error, 1e-6 over the change."""
    from paper_2403_17031_b200.pipeline import SFTStep
    N, K, V = 300, 64, 304
    E, W, mid, tokens, labels, mask = setup(N, K, V, False, seed=3)
    step = SFTStep(W, N, padding_id=-1, grad_dtype=F32)

    def f(E, W):
        h = (E[tokens.long()].float() @ mid.float()).to(BF16)
        return P.lmhead_xent(h, W, labels, mask=mask, want_dH=False, want_dW=False)["loss"].item()

    x = step.embed(E, tokens)
    h, back, _ = model(x, mid)
    o = step.loss(h, W, labels, mask)
    step.grad_embed(back(o["dH"]), tokens)
    for which, grad in ((1, o["dW"]), (0, o["dE"])):
        at = (E, W)[which].float()
        d = grad.float() * (0.05 * at.norm() / grad.float().norm())
        up, down = (at + d).to(BF16), (at - d).to(BF16)
        change = f(E, up) - f(E, down) if which else f(up, W) - f(down, W)
        told = ((up.double() - down.double()) * grad.double()).sum().item()
        assert abs(change - told) < 0.05 * abs(told), (which, change, told)


def test_a_captured_step_replays_on_new_data(P):
    from paper_2403_17031_b200.pipeline import SFTStep
    N, K, V = 600, 64, 1008
    E, W, mid, tokens, labels, mask = setup(N, K, V, False, seed=1)
    one, two = SFTStep(W, N, padding_id=1), SFTStep(W, N, padding_id=1)
    dmid = torch.empty(K, K, device="cuda")

    def run(step):
        x = step.embed(E, tokens)
        h, back, weight = model(x, mid)
        o = step.loss(h, W, labels, mask)
        dmid.copy_(weight(o["dH"]))
        step.grad_embed(back(o["dH"]), tokens)
        step.clip(0.01, [dmid])
        return o

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(one)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(one)
    E2, W2, _, tokens2, labels2, mask2 = setup(N, K, V, False, seed=2)
    for a, b in ((E, E2), (W, W2), (tokens, tokens2), (labels, labels2), (mask, mask2)):
        a.copy_(b)
    g.replay()
    torch.cuda.synchronize()
    got = {n: t.clone() for n, t in one.out.items()}
    want = run(two)
    assert all(torch.equal(got[n], want[n]) for n in got)
    assert one.device_status() == 0


def test_a_step_without_a_real_row(P):
    from paper_2403_17031_b200.pipeline import SFTStep
    E, W, mid, tokens, labels, mask = setup(50, 64, 304, False)
    step = SFTStep(W, 50, padding_id=1)
    step.embed(E, tokens)
    o = step.loss(step.out["hidden"], W, labels, torch.zeros_like(mask))
    step.grad_embed(o["dH"], tokens)
    assert float(o["loss"]) == 0 and step.clip(1.0).tolist() == [0.0, 1.0] and step.device_status() == 2


def test_a_longer_list_leaves_a_captured_clip_its_scratch(P):
    from paper_2403_17031_b200.pipeline import SFTStep
    E, W, mid, tokens, labels, mask = setup(50, 64, 304, False)
    step = SFTStep(W, 50, padding_id=1)
    fill = lambda: (step.out["dW"].fill_(1), step.out["dE"].fill_(1))                # noqa: E731
    fill()
    step.clip(1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.clip(1.0)
    scratch = next(iter(step._clip_scratch.values()))
    fill()
    step.clip(1.0, [torch.ones(3, device="cuda") for _ in range(1000)])
    assert any(t is scratch for t in step._clip_scratch.values())
    fill()
    graph.replay()
    n = step.out["dW"].numel() + step.out["dE"].numel()
    assert abs(step.out["norm"][0].item() / n ** 0.5 - 1) < 2.0 ** -22
