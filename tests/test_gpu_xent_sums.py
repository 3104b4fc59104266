"""ppo_lmhead_xent where the tensor cores' sums are exact, or nearly: what is given back for sums that were cut off must not be given to sums
that were not.

Tolerances. The logits z are exact. Base 2, y = z log2(e): the constant is rounded (2^-24 of y), y - reference is one rounding of at
most |y - reference| 2^-24, the exponential adds 2^-22, relative; lse adds up to 128 and then `chunks` of those in fp32, (128 + chunks + 8)
2^-23 in all, and three roundings of its size (reference + log2, times ln 2, with that rounded too); nll adds the label's product and its difference,
two more of the size of z and lse."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32
HALF, EPS = 2.0 ** -24, 2.0 ** -23


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


def stored(W, layout):
    return W if layout == "kv" else W.t().contiguous().t()


def check(o, H, W, labels):
    z = H.double() @ W.double()
    lse = torch.logsumexp(z, 1)
    at = z.gather(1, labels.long()[:, None])[:, 0]
    size, V = z.abs().amax(1), W.shape[1]
    sums = (128 + -(-V // 128) + 8) * EPS
    assert ((o["lse"].double() - lse).abs() <= sums + 2 * size * HALF + 3 * lse.abs() * HALF).all()
    assert ((o["nll"].double() - (lse - at)).abs() <= sums + 4 * size * HALF + 5 * (lse.abs() + (lse - at).abs()) * HALF).all()
    # and the header's reading of the two: their difference is the label's logit
    assert ((o["lse"] - o["nll"]).double() - at).abs().max() <= 2 * sums + (size * 6 + lse.abs() * 9 + (lse - at).abs() * 5).max() * HALF


@pytest.mark.parametrize("layout", ["kv", "vk"])
@pytest.mark.parametrize("M", [40, 100, 300])
@pytest.mark.parametrize("elements", [[0], [4095], [5, 2000], [0, 1, 2, 3, 16, 17]])
def test_few_elements_of_a_long_contraction(P, elements, M, layout):
    """All but a few hidden elements are 0: products with the same last places, whose sums are exact. Logits near -90 times
    the elements, 60 either way of that."""
    K, V = 4096, 3000
    g = torch.Generator().manual_seed(1)
    H, W = torch.zeros(M, K), torch.randn(K, V, generator=g)
    n = len(elements)
    H[:, elements] = 8.0
    W[elements] = (torch.randint(-60, 61, (n, V), generator=g) - 90.0) / 8               # products are whole numbers
    H, W = H.to(BF16).cuda(), stored(W.to(BF16).cuda(), layout)
    labels = torch.randint(0, V, (M,), generator=g, dtype=I32).cuda()
    check(P.lmhead_xent(H, W, labels), H, W, labels)


@pytest.mark.parametrize("layout", ["kv", "vk"])
@pytest.mark.parametrize("M", [40, 300])
def test_products_that_fp32_sums_exactly(P, M, layout):
    """Every hidden element counts, and every product is a multiple of 2^-4: sums are exact whatever their order. Logits of tens."""
    K, V = 4096, 3000
    g = torch.Generator().manual_seed(2)
    H = torch.randint(-2, 3, (M, K), generator=g).float()
    W = torch.randint(-2, 3, (K, V), generator=g).float() / 4
    H[:, 0], W[0] = 8.0, -8.0
    H, W = H.to(BF16).cuda(), stored(W.to(BF16).cuda(), layout)
    labels = torch.randint(0, V, (M,), generator=g, dtype=I32).cuda()
    check(P.lmhead_xent(H, W, labels), H, W, labels)


@pytest.mark.parametrize("K", [64, 1024, 1032, 2056])
@pytest.mark.parametrize("M", [40, 300])
def test_hidden_elements_that_are_zero_change_nothing(P, M, K):
    """The same rows with zeros behind them, in H or in W: the same bits."""
    V, more = 1000, 8192
    g = torch.Generator().manual_seed(3)
    H, W = torch.randn(M, K, generator=g).to(BF16).cuda(), (torch.randn(K, V, generator=g) * 3 / K ** 0.5).to(BF16).cuda()
    labels = torch.randint(0, V, (M,), generator=g, dtype=I32).cuda()
    want = P.lmhead_xent(H, W, labels)
    for h, w in ((0.0, 1.0), (1.0, 0.0), (0.0, 0.0)):
        H2, W2 = torch.full((M, more), h, dtype=BF16, device="cuda"), torch.full((more, V), w, dtype=BF16, device="cuda")
        H2[:, :K], W2[:K] = H, W
        o = P.lmhead_xent(H2, W2, labels)
        assert torch.equal(o["nll"], want["nll"]) and torch.equal(o["lse"], want["lse"])


@pytest.mark.parametrize("K", [4096, 16384, 65536])
def test_sums_that_are_cut_off_are_off_by_chance_only(P, K):
    """Dense values: every 16 elements 3/8 of a last place is cut off on average, 0.36 * 3 * 2^-26 of the logit in all for each of the K / 16 times.
    At least half of that mean is given back, whatever K, beside the constant's and the products' rounding, 2^-23."""
    M, V = 64, 1000
    g = torch.Generator().manual_seed(4)
    W = torch.randn(K, V, generator=g) / K ** 0.5
    H = torch.randn(M, K, generator=g)
    labels = torch.randint(0, V, (M,), generator=g, dtype=I32)
    H += 20.0 * W[:, labels.long()].t()                                                  # logits of 20 at the labels
    H, W, labels = H.to(BF16).cuda(), W.to(BF16).cuda(), labels.cuda()
    o = P.lmhead_xent(H, W, labels, want_dH=False, want_dW=False)
    z = (H.double() @ W.double()).gather(1, labels.long()[:, None])[:, 0]
    off = ((o["lse"] - o["nll"]).double() - z) / z
    print("K %d: mean %.3g, largest %.3g" % (K, off.mean(), off.abs().max()))
    assert off.mean().abs() <= 0.5 * 0.36 * 3 * 2.0 ** -26 * K / 16 + EPS
