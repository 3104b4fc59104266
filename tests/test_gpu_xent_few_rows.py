"""ppo_lmhead_xent's dW of up to 64 rows, whose H with the gradient's factor is not rounded to 16 bits.

In norm: the result's own rounding, taken from the definition's values; what the other roundings do (U and the factor for the label's element, half a
step of 2^-8 each) touches only elements away from the labels, and counts by their share of the gradient's norm. Sums of the two in squares,
with a tenth of that for fp32's sums and the chance of so many roundings."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


def make(M, K, V, layout, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    H = torch.randn(M, -(-K // 8) * 8, generator=g, device="cuda").to(BF16)[:, :K]
    shape = (K, V) if layout == "kv" else (V, K)
    W = (torch.randn(shape[0], -(-shape[1] // 8) * 8, generator=g, device="cuda") * (2 / K ** 0.5)).to(BF16)[:, :shape[1]]
    return H, W if layout == "kv" else W.t(), torch.randint(0, V, (M,), generator=g, device="cuda", dtype=I32)


@pytest.mark.parametrize("layout", ["kv", "vk"])
@pytest.mark.parametrize("M,K,V", [(1, 64, 5000), (2, 1032, 8003), (17, 264, 9000), (33, 77, 7001), (53, 520, 30011), (64, 100, 4099), (64, 1000, 20000)])
def test_weight_gradient(P, M, K, V, layout):
    H, W, labels = make(M, K, V, layout)
    mask = (torch.arange(M, device="cuda") % 7 != 3).to(torch.uint8)
    o = P.lmhead_xent(H, W, labels, mask=mask, temperature=0.7, scale=3.0)
    real, at, tau = mask.double(), labels.long()[:, None], float(torch.tensor(0.7))
    n = int(real.sum())
    D = torch.softmax(H.double() @ W.double() / tau, 1)
    D.scatter_add_(1, at, torch.full_like(at, -1, dtype=D.dtype))
    D *= 3.0 * real[:, None] / (n * tau)
    want = H.double().t() @ D
    away = (H.double().t() @ D.scatter(1, at, 0.0)).norm() / want.norm()
    rounding = (want.to(BF16).double() - want).norm() / want.norm()
    off = ((o["dW"].double() - want).norm() / want.norm()).item()
    assert off <= 1.1 * (rounding ** 2 + (away * 2 * 2.0 ** -8) ** 2) ** 0.5, (off, rounding, away)


@pytest.mark.parametrize("M", [1, 50, 64, 128])
def test_factors_beyond_the_range(P, M):
    """A power of two as scale changes no digit; a factor that makes a H infinite leaves no finite gradient, and none that looks like one."""
    H, W, labels = make(M, 64, 1000, "kv", seed=1)
    want = P.lmhead_xent(H, W, labels)["dW"].double()
    got = P.lmhead_xent(H, W, labels, scale=2.0 ** 100)["dW"].double() * 2.0 ** -100
    assert torch.isfinite(got).all() and torch.equal(got, want)
    for denom in (0.0, 1e-45):
        o = P.lmhead_xent(H, W, labels, denom=torch.tensor([denom], device="cuda"))
        assert not torch.isfinite(o["dW"]).any() and not torch.isfinite(o["loss"])


@pytest.mark.parametrize("withhold", [1, 2], ids=["finished", "drained"])
def test_waits_that_run_out_are_nan_and_reported(P, tmp_path_factory, withhold):
    """A copy of the call whose finished (1) or drained (2) accumulators are never announced, and whose waits are short: it ends, says so, and
    returns NaN; the library then works on the same buffers."""
    import ctypes as C
    import os
    from paper_2403_17031_b200 import binding, build
    path = build.build_variant(os.path.join(str(tmp_path_factory.mktemp("xent")), "libxent_few%d.so" % withhold),
                               ["PPO_TEST_WITHHOLD_XENT=%d" % withhold, "PPO_TC_WAIT_TRIES=32768"], only=["ppo_lmhead_xent.cu"])
    fn = C.CDLL(path).ppo_lmhead_xent
    fn.restype, fn.argtypes = binding._SIGS["ppo_lmhead_xent"]
    p = lambda t: C.c_void_p(t.data_ptr())                                          # noqa: E731
    M, K, V = 53, 512, 50304                             # more than two tiles of every product for a worker
    H, W, labels = make(M, K, V, "kv")
    scratch = torch.empty(P.lmhead_xent_scratch_bytes(M, K, V), dtype=torch.uint8, device="cuda")
    out = {"loss": torch.zeros((), device="cuda"), "nll": torch.zeros(M, device="cuda"), "lse": torch.zeros(M, device="cuda"),
           "dH": torch.zeros_like(H), "dW": torch.zeros_like(W)}
    ws = P.new_workspace(256)
    assert fn(p(H), K, p(W), V, 0, M, K, V, p(labels), None, -100, 1.0, 1.0, None, 0, p(out["loss"]), p(out["nll"]), p(out["lse"]), p(out["dH"]), K,
              p(out["dW"]), V, p(ws), p(scratch), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    assert all(torch.isnan(t).all() for t in out.values()) and P.last_device_status(ws) & 4
    P.lmhead_xent(H, W, labels, workspace=ws, scratch=scratch, out=out)
    want = P.lmhead_xent(H, W, labels)
    assert P.last_device_status(ws) == 0 and all(torch.equal(out[n], want[n]) and torch.isfinite(out[n]).all() for n in out)
