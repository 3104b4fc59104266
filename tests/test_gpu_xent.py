"""ppo_lmhead_xent against oracle/sft_oracle.py.

Tolerances, element by element. A logit is a sum of K products in fp32, each addition off by at most 2^-23 of its absolute partial sum
(rounded or cut off): ez = (K + 4) 2^-23 max_j sum_k |h_k w_kj| / tau, and its scaling to base 2 adds 2^-23 of its size. The log-sum-exp
moves by at most the largest of these; its own sum of up to 128 exponentials (2^-22 each), joined over the chunks, adds less than
(128 + chunks) 2^-23. U is off by those, relative, and by half a step of bf16 (2^-8); the sum of the rounded U, which divides it, by another
half step at most: two in the worst case, and as much for 1 - p at the label; the factor that makes U at the label exact adds one to the others.
In dW a H adds another. In dH, c times a mean of columns of W adds at most half a step of D at the label times the row's largest |w|. Results
are off by half a step of their own; the products over V columns or M rows by (V + 4) 2^-23 and
(M + 4) 2^-23 of the sums of the absolute products."""
import numpy as np
import pytest
import torch

from oracle import sft_oracle as O
from parity import npy

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
STEP, EPS = 2.0 ** -8, 2.0 ** -23


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


def make(M, K, V, layout="kv", seed=0, size=1.0, pad=0):
    """H [M, K] with a row pitch, W [K, V] stored by rows or by columns with a pitch of a multiple of 8, labels."""
    g = torch.Generator().manual_seed(seed)
    up = lambda n: -(-n // 8) * 8 + pad                                               # noqa: E731
    H = torch.full((M, up(K)), 7.0, dtype=BF16, device="cuda")[:, :K]
    H.copy_(torch.randn(M, K, generator=g))
    shape = (K, V) if layout == "kv" else (V, K)
    W = torch.full((shape[0], up(shape[1])), 7.0, dtype=BF16, device="cuda")[:, :shape[1]]
    W.copy_(torch.randn(*shape, generator=g) * (size / K ** 0.5))
    labels = torch.randint(0, V, (M,), generator=g, dtype=I32).cuda()
    return H, W if layout == "kv" else W.t(), labels


def check(o, H, W, labels, real, tau, scale=1.0, denom=None, least=0.0):
    """Compares a call's results with the definition; returns the oracle's. least: a probability that the gradients may take for 0."""
    h, w, real = f64(H), f64(W), np.asarray(real) != 0
    want = O.xent(h, w, npy(labels), real, tau, scale, denom)
    (M, K), V = h.shape, w.shape[1]
    z = h @ w / np.float64(np.float32(tau))
    ez = ((K + 4) * EPS * (np.abs(h) @ np.abs(w)).max(1) / tau + np.abs(z).max(1) * 2 * EPS) * real
    es = (128 + -(-V // 128) + 8) * EPS
    lse_tol = ez + es + np.abs(want["lse"]) * 4 * EPS
    assert (np.abs(f64(o["lse"]) - want["lse"]) <= lse_tol).all()
    nll_tol = 2 * ez + es + (np.abs(want["lse"]) + np.abs(want["nll"])) * 4 * EPS
    assert (np.abs(f64(o["nll"]) - want["nll"]) <= nll_tol).all()
    d = denom if denom is not None else max(1, real.sum())
    assert abs(float(o["loss"]) - want["loss"]) <= nll_tol.sum() / d + abs(want["loss"]) * EPS
    assert not f64(o["nll"])[~real].any() and not f64(o["lse"])[~real].any()
    # p is off by twice the logits' error; at the label it is 1 - p that counts, off by that much of p
    D, er = np.abs(want["D"]), (2 * ez + 2 * es)[:, None]
    p = D * er + least * abs(scale) / (d * tau) * real[:, None]
    for r in np.flatnonzero(real):
        p[r, npy(labels)[r]] = abs(scale) / (d * tau) * er[r, 0]
    tiny = 2.0 ** -120
    if o["dH"] is not None:
        at = np.clip(npy(labels), 0, V - 1)
        tol = (3 * STEP * D + p) @ np.abs(w).T + (V + 4) * EPS * (D @ np.abs(w).T) + STEP * np.abs(want["dH"]) + tiny
        tol += STEP * D[np.arange(M), at][:, None] * np.abs(w).max(1)
        assert (np.abs(f64(o["dH"]) - want["dH"]) <= 1.01 * tol).all()
        assert not f64(o["dH"])[~real].any()
    if o["dW"] is not None:
        ah = np.abs(h) * real[:, None]
        tol = ah.T @ (4 * STEP * D + p) + (M + 4) * EPS * (ah.T @ D) + STEP * np.abs(want["dW"]) + tiny
        assert (np.abs(f64(o["dW"]) - want["dW"]) <= 1.01 * tol).all()
    return want


@pytest.mark.parametrize("layout", ["kv", "vk"])
@pytest.mark.parametrize("M,K,V", [(1, 64, 256), (3, 8, 2), (53, 256, 1000), (257, 72, 1003), (300, 33, 515), (130, 520, 4099), (600, 128, 130),
                                   (5, 1024, 20000)])
def test_matches_the_definition(P, M, K, V, layout):
    H, W, labels = make(M, K, V, layout, pad=8)
    o = P.lmhead_xent(H, W, labels, temperature=0.7)
    check(o, H, W, labels, np.ones(M), 0.7)
    assert o["dW"].stride(1 if layout == "kv" else 0) == 1


@pytest.mark.parametrize("layout", ["kv", "vk"])
@pytest.mark.parametrize("M,piece", [(700, 256), (1024, 512), (513, 256), (700, 0)])
def test_masked_and_ignored_rows_in_pieces(P, M, piece, layout):
    H, W, labels = make(M, 136, 777, layout, seed=1)
    mask = (torch.rand(M, generator=torch.Generator().manual_seed(2)) > 0.4).to(torch.uint8).cuda()
    labels[::5] = -100
    ws = P.new_workspace(P.workspace_bytes(M, 1, 777))
    o = P.lmhead_xent(H, W, labels, mask=mask, piece_rows=piece, workspace=ws, scale=2.0)
    check(o, H, W, labels, npy(mask) * (npy(labels) != -100), 1.0, scale=2.0)
    assert P.last_device_status(ws) == 0


@pytest.mark.parametrize("left", [0, 1, 256, 257])
def test_few_real_rows_of_several_pieces(P, left):
    """Pieces without a row, a piece of one row, and none at all."""
    M = 1000
    H, W, labels = make(M, 64, 300, seed=3)
    mask = torch.zeros(M, dtype=torch.uint8, device="cuda")
    mask[torch.randperm(M, generator=torch.Generator().manual_seed(1))[:left].cuda()] = 1
    ws = P.new_workspace(P.workspace_bytes(M, 1, 300))
    o = P.lmhead_xent(H, W, labels, mask=mask, piece_rows=256, workspace=ws)
    check(o, H, W, labels, npy(mask), 1.0)
    assert P.last_device_status(ws) == (0 if left else 2)
    if not left:
        assert float(o["loss"]) == 0 and not o["dW"].any() and not o["dH"].any()


@pytest.mark.parametrize("shift", [-300.0, 90.0, 2000.0])
def test_logits_far_from_zero(P, shift):
    H, W, labels = make(200, 64, 1500, seed=4)
    H[:, 0] = 4
    W[0] = shift / 4
    check(P.lmhead_xent(H, W, labels), H, W, labels, np.ones(200), 1.0)


@pytest.mark.parametrize("layout", ["kv", "vk"])
def test_what_all_columns_share_drops_out(P, layout):
    """sum_j D_j = 0: a row of W that is the same in all columns gets no gradient through H but what fp32 leaves: the sums of V and of the row's
    products, the rounded sum that divides them and the label's part, (2 V + 16) 2^-23 of sum |D| |w| in all."""
    H, W, labels = make(200, 64, 3000, layout, seed=16)
    H[:, 0] = 8
    W[0] = -11.25
    o = P.lmhead_xent(H, W, labels)
    want = check(o, H, W, labels, np.ones(200), 1.0)
    assert (np.abs(f64(o["dH"][:, 0])) <= 11.25 * np.abs(want["D"]).sum(1) * (2 * 3000 + 16) * EPS).all()


def test_columns_of_different_sizes(P):
    """Chunks of columns whose largest logits lie hundreds apart have references of their own."""
    H, W, labels = make(200, 64, 1500, "vk", seed=5)
    H[:, 0] = 4
    W[0] = ((torch.arange(1500) // 100) % 5 * 40.0 - 90).to(BF16).cuda()
    check(P.lmhead_xent(H, W, labels), H, W, labels, np.ones(200), 1.0)


def test_confident_rows(P):
    """1 - p at the label is small: the gradient there is taken without cancelling more than fp32 does."""
    H, W, labels = make(100, 128, 1000, seed=6)
    H += 3.0 * W[:, labels.long()].t() * 16
    check(P.lmhead_xent(H, W, labels), H, W, labels, np.ones(100), 1.0)


def test_tiles_cut_along_the_vocabulary(P):
    """Few tiles of dH and a long vocabulary: several pairs of blocks share a tile."""
    H, W, labels = make(300, 264, 30011, "vk", seed=7)
    check(P.lmhead_xent(H, W, labels), H, W, labels, np.ones(300), 1.0)


def test_loss_alone_one_gradient_alone_and_denominator(P):
    H, W, labels = make(150, 64, 700, seed=8)
    both = P.lmhead_xent(H, W, labels)
    for dh, dw in ((False, False), (True, False), (False, True)):
        o = P.lmhead_xent(H, W, labels, want_dH=dh, want_dW=dw)
        for name in ("loss", "nll", "lse", "dH", "dW"):
            assert o[name] is None if name == ("dH" if not dh else "") or name == ("dW" if not dw else "") else torch.equal(o[name], both[name])
    denom = torch.tensor([37.0], device="cuda")
    check(P.lmhead_xent(H, W, labels, denom=denom, scale=0.5), H, W, labels, np.ones(150), 1.0, 0.5, 37.0)


def test_bad_labels_and_a_nan_row(P):
    H, W, labels = make(40, 64, 500, seed=9)
    ws = P.new_workspace(P.workspace_bytes(40, 1, 500))
    labels[3], labels[30] = 500, -1
    o = P.lmhead_xent(H, W, labels, workspace=ws)
    assert P.last_device_status(ws) == 1 and torch.isnan(o["loss"]) and torch.isnan(o["dW"]).all()
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[3, 30]] = True
    assert torch.isnan(o["nll"][bad]).all() and torch.isnan(o["dH"][bad]).all()
    want = O.xent(f64(H), f64(W), npy(labels), np.ones(40), 1.0)
    assert np.abs(f64(o["nll"])[~npy(bad)] - want["nll"][~npy(bad)]).max() < 1e-4 and torch.isfinite(o["dH"][~bad]).all()
    H, W, labels = make(40, 64, 500, seed=9)
    H[7, 5] = torch.nan
    o = P.lmhead_xent(H, W, labels)
    rest = torch.arange(40, device="cuda") != 7
    assert torch.isnan(o["nll"][7]) and torch.isfinite(o["nll"][rest]).all() and torch.isfinite(o["dH"][rest]).all()
    mask = rest.to(torch.uint8)                                       # left out, it harms nobody
    check(P.lmhead_xent(H.nan_to_num(), W, labels, mask=mask), H.nan_to_num(), W, labels, npy(mask), 1.0)
    o = P.lmhead_xent(H, W, labels, mask=mask)
    assert torch.isfinite(o["dW"]).all() and torch.isfinite(o["loss"]) and not o["dH"][7].any()


@pytest.mark.parametrize("layout", ["kv", "vk"])
@pytest.mark.parametrize("pitch", [0, 3, 8])
def test_elements_behind_rows_are_left_alone(P, pitch, layout):
    M, K, V = 270, 70, 523
    H, W, labels = make(M, K, V, layout, seed=10)
    dH = torch.full((M, K + pitch), 3.0, dtype=BF16, device="cuda")
    shape = (K, V) if layout == "kv" else (V, K)
    dW = torch.full((shape[0] + 1, shape[1] + pitch), 3.0, dtype=BF16, device="cuda")
    out = {"loss": torch.empty((), device="cuda"), "nll": torch.empty(M, device="cuda"), "lse": torch.empty(M, device="cuda"),
           "dH": dH[:, :K], "dW": dW[:-1, :shape[1]] if layout == "kv" else dW[:-1, :shape[1]].t()}
    o = P.lmhead_xent(H, W, labels, out=out)
    check(o, H, W, labels, np.ones(M), 1.0)
    assert (dH[:, K:] == 3).all() and (dW[:, shape[1]:] == 3).all() and (dW[-1] == 3).all()


def test_same_bits_on_another_stream_in_a_graph_and_beside_another_call(P):
    H, W, labels = make(600, 200, 3000, seed=11)
    H2, W2, labels2 = make(600, 200, 3000, seed=12)
    mask = (torch.rand(600, generator=torch.Generator().manual_seed(2)) > 0.3).to(torch.uint8).cuda()
    names = ("loss", "nll", "lse", "dH", "dW")
    one, two = P.lmhead_xent(H, W, labels, mask=mask, piece_rows=256), P.lmhead_xent(H2, W2, labels2)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        a = P.lmhead_xent(H, W, labels, mask=mask, piece_rows=256)
    with torch.cuda.stream(t):
        b = P.lmhead_xent(H2, W2, labels2)
    torch.cuda.synchronize()
    assert all(torch.equal(a[n], one[n]) and torch.equal(b[n], two[n]) for n in names)
    scratch = torch.empty(P.lmhead_xent_scratch_bytes(600, 200, 3000, 256), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = P.lmhead_xent(H, W, labels, mask=mask, piece_rows=256, scratch=scratch)
    scratch.fill_(255)
    g.replay()
    assert all(torch.equal(o[n], one[n]) for n in names)
    H.copy_(H2)
    labels.copy_(labels2)
    mask.fill_(1)
    g.replay()
    want = P.lmhead_xent(H2, W, labels2, mask=mask, piece_rows=256)
    assert all(torch.equal(o[n], want[n]) for n in names)


def test_agrees_with_the_log_prob_calls(P):
    """The same quantities as ppo_lmhead_logprob_entropy and ppo_lmhead_bwd, which form the logits on other tiles."""
    M, K, V = 384, 256, 5000
    H, W, labels = make(M, K, V, seed=13)
    H, W = H.contiguous(), W.contiguous()
    ws = P.new_workspace(P.lmhead_workspace_bytes(M, K, V))
    lp, _, lse = P.lmhead_logprob_entropy(H, W, labels, 0.7, ws)
    o = P.lmhead_xent(H, W, labels, temperature=0.7)
    assert (o["nll"] + lp).abs().max() < 1e-4 and (o["lse"] - lse).abs().max() < 1e-4
    back = P.lmhead_bwd(H, W, labels, lse, torch.full((M,), -1.0 / M, device="cuda"), 0.7, ws)
    dH, dW = back["dH"], back["dW"]
    assert ((o["dH"].float() - dH.float()).norm() / dH.float().norm() < 2 * STEP)
    assert ((o["dW"].float() - dW.float()).norm() / dW.float().norm() < 2 * STEP)


def test_no_rows(P):
    H, W, labels = make(1, 64, 300, seed=14)
    o = P.lmhead_xent(H[:0], W, labels[:0])
    torch.cuda.synchronize()
    assert float(o["loss"]) == 0 and not o["dW"].any() and o["dH"].shape == (0, 64)


def test_refuses_what_it_does_not_take(P):
    H, W, labels = make(8, 64, 300, seed=15)
    with pytest.raises(P.PPOError):
        P.lmhead_xent(H, W[:, :299].contiguous(), labels)             # rows of W that are no multiple of 16 bytes
    with pytest.raises(ValueError):
        P.lmhead_xent(H, W, labels[:5])
    with pytest.raises(TypeError):
        P.lmhead_xent(H, W.float(), labels)
    with pytest.raises(ValueError):
        P.lmhead_xent(H, W, labels, scratch=torch.empty(256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("kind", ["first", "last", "four", "even"])
@pytest.mark.parametrize("shift", [-90.0, 40.0])
def test_lse_of_logits_far_from_zero(P, kind, shift):
    """The tensor cores cut their sums off after every 16 elements: at K = 4096 that is 256 times 3/8 of 2^-17 on average for sums between
    64 and 128, 7.3e-4 in all where one element brings the sum there. What is common to a row's logits is given back to lse. Left is the
    chance of single cuts (0 to 3 quarters of 2^-17, each 0.28 2^-17 off the mean: 16 * 0.28 * 2^-17 = 3.4e-5 for a column; five times that), what the factor on the logits
    adds for columns up to 15 above the mean (3.4e-6 15 = 5e-5), and four roundings of 90 in fp32 (4.3e-5): 2.6e-4."""
    M, K, V = 40, 4096, 3000
    g = torch.Generator().manual_seed(11)
    H, W = torch.randn(M, K, generator=g), torch.randn(K, V, generator=g) * (3 / K ** 0.5)
    at = {"first": [0], "last": [K - 1], "four": [0, 700, 1400, 2100]}.get(kind)
    if at:
        H[:, at], W[at] = 8.0, shift / 8 / len(at)
    else:
        H, W = H + 1, W + shift / K
    H, W = H.to(BF16).cuda(), W.to(BF16).cuda()
    labels = torch.randint(0, V, (M,), generator=g, dtype=I32).cuda()
    o = P.lmhead_xent(H, W, labels, want_dH=False, want_dW=False)
    want = torch.logsumexp(H.double() @ W.double(), 1)
    assert (o["lse"].double() - want).abs().max() <= 2.6e-4


@pytest.mark.parametrize("layout", ["kv", "vk"])
@pytest.mark.parametrize("M,K,V", [(2, 1, 135), (70, 1, 135), (300, 1, 3), (5, 1, 1), (4, 40, 1), (200, 9, 1)])
def test_sizes_of_one(P, M, K, V, layout):
    H, W, labels = make(M, K, V, layout, seed=17)
    before = W.clone()
    o = P.lmhead_xent(H, W, labels)
    check(o, H, W, labels, np.ones(M), 1.0)
    assert torch.equal(W, before) and o["dW"].shape == (K, V)


@pytest.mark.parametrize("M", [1, 26, 100, 300])
@pytest.mark.parametrize("layout", ["kv", "vk"])
def test_columns_beside_the_largest_with_a_reference_of_their_own(P, M, layout):
    """Logits 2^y with a row's mean at 0: the sampled columns and their reference lie there, the largest values at the edges of what it
    serves (base 2: -32 to 96) and 128 from there, in chunks beside one another: each of them counts."""
    H, W, labels = make(M, 64, 1500, layout, seed=18)
    H.zero_()
    H[:, 0], H[:, 1] = 8.0, 0.25
    base = torch.zeros(1500, dtype=torch.float64)
    for chunk, y in enumerate((95.5, 96.5, 97.0, 95.0, -40.0, 96.0, 97.5)):
        base[128 * chunk + 5] = y
        base[128 * chunk + 77] = y - 1
    W[0] = (base * float(np.log(2.0)) / 8).to(BF16).cuda()
    labels[::3] = 133
    check(P.lmhead_xent(H, W, labels), H, W, labels, np.ones(M), 1.0)


@pytest.mark.parametrize("V", [300, 513, 576, 577, 640])
@pytest.mark.parametrize("M", [5, 100, 300])
@pytest.mark.parametrize("y", [-200.0, 120.0, 200.0])
def test_the_last_columns_lie_far_from_the_others(P, M, V, y):
    """One to 128 columns in the last chunk, with logits 2^y of their own; the largest ones, or the smallest. A row's largest U is 2^-64 at
    least, and what is under 2^-126 beside it becomes 0: a probability of 2^-62."""
    H, W, labels = make(M, 64, V, "vk", seed=19)
    H[:, 0] = 8.0
    W[0, :(V - 1) // 128 * 128] = 0
    W[0, (V - 1) // 128 * 128:] = y * float(np.log(2.0)) / 8
    labels[::3] = V - 1
    check(P.lmhead_xent(H, W, labels), H, W, labels, np.ones(M), 1.0, least=2.0 ** -62)
