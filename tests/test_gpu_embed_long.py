"""ppo_embed_bwd where counts are summed by a launch of their own (more than 262144 positions), where chunks hold 64 and 128 entries, and where
few positions have too many tokens to be ranked (2^19 and more) -- against sums in 64 bits on the device.

n summands in fp32, each addition off by at most 2^-24 of its partial sum, the scale one more, what is added to one more; then half a step of the
type."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


SIZES = [(262144, 8, 50277), (262145, 8, 50277), (300001, 40, 300), (700000, 5, 65536), (300000, 8, 1 << 19),          # counts summed
         (120001, 4096, 2000), (250001, 4096, 50304),                                                               # chunks of 64, of 128
         (129, 24, 1 << 19), (5000, 24, (1 << 19) + 3), (8192, 8, 1 << 20), (5000, 9, (1 << 19) - 1), (3000, 4, (1 << 24) + 5)]   # three and four passes


@pytest.mark.parametrize("N,K,V", SIZES)
@pytest.mark.parametrize("out,accumulate", [(F32, False), (BF16, False), (F32, True)])
def test_gradient(P, N, K, V, out, accumulate):
    g = torch.Generator(device="cuda").manual_seed(N)
    dY = torch.randn(N, K, generator=g, device="cuda").to(BF16)
    # ids of which a few make up most, one of them a third, and the last ones
    tokens = (torch.rand(N, generator=g, device="cuda", dtype=torch.float64) ** 6 * V).to(I32).clamp(max=V - 1)
    tokens[torch.rand(N, generator=g, device="cuda") < 0.33] = 7
    tokens[-3:] = torch.tensor([V - 1, V - 2, V - 1], dtype=I32)
    tokens[::50] = 1
    base = torch.randn(V, K, generator=g, device="cuda").to(out) if accumulate else torch.full((V, K), 9.0, dtype=out, device="cuda")
    got = base.clone()
    ws = P.new_workspace(256)
    P.embed_bwd(dY, tokens, V, scale=0.5, padding_id=1, out=got, accumulate=accumulate, workspace=ws)
    assert P.last_device_status(ws) == 0
    at = tokens.long()
    counts = torch.bincount(at, minlength=V)
    counts[1] = 0
    kept = (at != 1).nonzero()[:, 0]
    for c in range(0, K, 256):
        x = dY[:, c:c + 256][kept].double()
        want = torch.zeros(V, x.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at[kept], x) * 0.5
        size = torch.zeros_like(want).index_add_(0, at[kept], x.abs()) * 0.5
        b = base[:, c:c + 256].double() if accumulate else 0
        want = want + b
        tol = (counts[:, None] + 2) * 2.0 ** -24 * (size + (b.abs() if accumulate else 0)) + HALF[out] * want.abs()
        o = got[:, c:c + 256].double()
        assert ((o - want).abs() <= 1.01 * tol).all()
        assert torch.equal(o[counts == 0], b[counts == 0] if accumulate else torch.zeros_like(o[counts == 0]))
