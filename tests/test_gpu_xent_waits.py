"""ppo_lmhead_xent when a wait inside its products runs out. The only harmless way to make one do so: a second copy of the call is compiled in
which finished (1) or drained (2) accumulators are never announced, and in which waits are short. The call ends, reports it, everything it
returns is NaN, and the product library then works on the same buffers."""
import ctypes as C
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV_TIMEOUT = 4


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


@pytest.mark.parametrize("withhold", [1, 2], ids=["finished", "drained"])
def test_a_call_whose_waits_run_out_is_nan_and_reported(P, tmp_path_factory, withhold):
    from paper_2403_17031_b200 import binding, build
    path = build.build_variant(os.path.join(str(tmp_path_factory.mktemp("xent")), "libxent_withhold%d.so" % withhold),
                               ["PPO_TEST_WITHHOLD_XENT=%d" % withhold, "PPO_TC_WAIT_TRIES=32768"], only=["ppo_lmhead_xent.cu"])
    fn = C.CDLL(path).ppo_lmhead_xent
    fn.restype, fn.argtypes = binding._SIGS["ppo_lmhead_xent"]
    g = torch.Generator(device="cuda").manual_seed(5)
    p = lambda t: C.c_void_p(t.data_ptr()) if t is not None else None             # noqa: E731
    # blocks alone, pairs, wide tiles; in each a worker has more than two tiles of the first product, which every row needs
    for M, K, V in ((100, 128, 50304), (300, 128, 50304), (4864, 4096, 4096)):
        H = torch.randn(M, K, generator=g, device="cuda").bfloat16()
        W = (torch.randn(K, V, generator=g, device="cuda") / K ** 0.5).bfloat16()
        labels = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
        scratch = torch.empty(P.lmhead_xent_scratch_bytes(M, K, V), dtype=torch.uint8, device="cuda")
        out = {"loss": torch.zeros((), device="cuda"), "nll": torch.zeros(M, device="cuda"), "lse": torch.zeros(M, device="cuda"),
               "dH": torch.zeros_like(H), "dW": torch.zeros_like(W)}
        ws = P.new_workspace(256)
        st = C.c_void_p(torch.cuda.current_stream().cuda_stream)
        for status in (ws, None):
            for t in out.values():
                t.zero_()
            assert fn(p(H), K, p(W), V, 0, M, K, V, p(labels), None, -100, 1.0, 1.0, None, 0, p(out["loss"]), p(out["nll"]), p(out["lse"]),
                      p(out["dH"]), K, p(out["dW"]), V, p(status), p(scratch), st) == 0
            torch.cuda.synchronize()
            assert all(torch.isnan(t).all() for t in out.values()), (M, {n: int(torch.isnan(t).sum()) for n, t in out.items()})
        assert P.last_device_status(ws) & DEV_TIMEOUT
        P.lmhead_xent(H, W, labels, workspace=ws, scratch=scratch, out=out)
        assert P.last_device_status(ws) == 0
        want = P.lmhead_xent(H, W, labels)
        assert all(torch.equal(out[n], want[n]) and torch.isfinite(out[n]).all() for n in out)
