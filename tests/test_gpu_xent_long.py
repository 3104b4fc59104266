"""ppo_lmhead_xent at sizes whose gradients go through 256 x 512 tiles (a contraction of 4096 and more, two tiles and more for each pair of blocks),
against the definition in 64 bits on the device.

Element by element the tolerances are those of sums whose roundings all go one way: U half a step of bf16 (2^-8), the sum that divides it
another, the factor for the label's element one more, in dW a H another, the result one; products over V columns or M rows in fp32, (n + 4) 2^-23. Such
sums hide a tile that lies in another's place, so blocks of 128 x 128 are compared in norm as well: roundings are as often up as down there, so
that four of at most 2^-8 are well under 2^-7 together, and a block in another's place is off by more than its own norm."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32
STEP, EPS = 2.0 ** -8, 2.0 ** -23


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


def near(got, want, tol):
    d = (got.double() - want).abs()
    assert (d <= 1.01 * tol).all()
    pad = [0, -want.shape[1] % 128, 0, -want.shape[0] % 128]
    blocks = lambda t: torch.nn.functional.pad(t, pad).unflatten(1, (-1, 128)).unflatten(0, (-1, 128)).square().sum((1, 3)).sqrt()     # noqa: E731
    assert (blocks(d) <= 2 * STEP * blocks(want)).all()


@pytest.mark.parametrize("layout", ["kv", "vk"])
@pytest.mark.parametrize("M,piece", [(4900, 0), (9500, 4864)], ids=["one piece", "two pieces, rows left out"])
def test_wide_tiles(P, M, piece, layout):
    K, V, tau = 4096, 4997, 0.7
    g = torch.Generator(device="cuda").manual_seed(M)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")                   # noqa: E731
    H = rand(M, K).to(BF16)
    shape = (K, V) if layout == "kv" else (V, K)
    W = torch.full((shape[0], -(-shape[1] // 8) * 8), 7.0, dtype=BF16, device="cuda")[:, :shape[1]]
    W.copy_(rand(*shape) / K ** 0.5)
    W = W if layout == "kv" else W.t()
    labels = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=I32)
    mask = None
    real = torch.ones(M, dtype=torch.bool, device="cuda")
    if piece:
        real = torch.rand(M, generator=g, device="cuda") > 0.2
        mask = real.to(torch.uint8)
    ws = P.new_workspace(256)
    o = P.lmhead_xent(H, W, labels, mask=mask, temperature=tau, piece_rows=piece, workspace=ws)
    assert P.last_device_status(ws) == 0
    h, w, at, n = H.double() * real[:, None], W.double(), labels.long()[:, None], int(real.sum())
    z = h @ w / float(torch.tensor(tau))
    lse = torch.logsumexp(z, 1) * real
    nll = (lse - z.gather(1, at)[:, 0]) * real
    ez = (K + 4) * EPS * (h.abs() @ w.abs()).amax(1) / tau + z.abs().amax(1) * 2 * EPS
    es = (128 + -(-V // 128) + 8) * EPS
    assert ((o["lse"].double() - lse).abs() <= ez + es + lse.abs() * 4 * EPS).all()
    assert ((o["nll"].double() - nll).abs() <= 2 * ez + es + (lse.abs() + nll.abs()) * 4 * EPS).all()
    D = torch.softmax(z, 1)
    D.scatter_add_(1, at, torch.full_like(at, -1, dtype=D.dtype))
    D *= real[:, None] / (n * tau)
    er = 2 * ez + 2 * es
    size = D.abs()
    p = size * er[:, None]
    p.scatter_(1, at, (er * real / (n * tau))[:, None])
    want = D @ w.t()
    aw = w.abs().t()
    tol = (3 * STEP * size + p) @ aw + (V + 4) * EPS * (size @ aw) + STEP * want.abs() + 2.0 ** -120
    tol += STEP * size.gather(1, at) * w.abs().amax(1)
    assert not o["dH"][~real].any()
    near(o["dH"], want, tol)
    want = h.t() @ D
    tol = h.abs().t() @ (4 * STEP * size + p) + (M + 4) * EPS * (h.abs().t() @ size) + STEP * want.abs() + 2.0 ** -120
    near(o["dW"], want, tol)
