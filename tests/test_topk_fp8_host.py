"""Refusals of the alternatives, quantisation and 8-bit product calls: the documented codes, before any launch (no GPU)."""
import ctypes as C

import pytest
import torch

FAKE = 0x10000   # a non-null, 256-byte aligned address that is never dereferenced on these paths
P = C.c_void_p


@pytest.fixture(scope="module")
def b():
    from paper_2403_17031_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _codes(fn, ok, cases):
    for at, value, code in cases:
        args = list(ok)
        args[at] = value
        assert fn(*args) == code, (at, value, code)


def test_topk_refusals(b):
    # logits dtype rows V stride | tokens n mask temperature k | logprob entropy lse top_ids top_logprob ws stream
    ok = [P(FAKE), b.PPO_BF16, 4, 1000, 1000, P(FAKE), 1, None, 0.7, 5, P(FAKE), None, None, P(FAKE), P(FAKE), None, None]
    _codes(b.lib().ppo_logprob_topk, ok, [
        (1, 7, -5), (2, -1, -2), (2, 1 << 31, -2), (3, 0, -2), (3, 1 << 31, -2), (4, 999, -2), (6, -1, -2), (6, 129, -2),
        (9, -1, -2), (9, 129, -2), (8, 0.0, -3), (8, float("nan"), -3), (8, float("inf"), -3), (0, None, -1), (5, None, -1),
        (10, None, -1), (13, None, -1), (14, None, -1), (0, P(FAKE + 1), -4), (2, 0, 0)])
    few = list(ok)
    few[3] = few[4] = 4                                  # k above the vocabulary
    assert b.lib().ppo_logprob_topk(*few) == -2


def test_topk_bwd_refusals(b):
    # logits dtype rows V stride | tokens n dlogprob | top_ids k dtop | lse entropy dentropy dlse mask temperature | dlogits stride ws stream
    ok = [P(FAKE), b.PPO_F32, 4, 1000, 1000, P(FAKE), 1, P(FAKE), P(FAKE), 5, P(FAKE), P(FAKE), P(FAKE), P(FAKE), None, None, 0.7,
          P(2 * FAKE), 1000, None, None]
    _codes(b.lib().ppo_logprob_topk_bwd, ok, [
        (1, 7, -5), (2, -1, -2), (3, 0, -2), (4, 999, -2), (18, 999, -2), (6, 129, -2), (9, 129, -2), (6, -1, -2), (16, -1.0, -3),
        (0, None, -1), (17, None, -1), (11, None, -1), (5, None, -1), (7, None, -1), (8, None, -1), (10, None, -1),
        (12, None, -1),                                  # a gradient on the entropy needs the entropy
        (17, P(FAKE), -3), (0, P(FAKE + 2), -4), (17, P(2 * FAKE + 2), -4), (2, 0, 0)])


def test_quantize_refusals(b):
    # x dtype R C stride transpose block_rows | q stride scales stream
    ok = [P(FAKE), b.PPO_BF16, 64, 256, 256, 0, 1, P(FAKE), 256, P(FAKE), None]
    _codes(b.lib().ppo_fp8_quantize, ok, [
        (1, 2, -5), (2, -1, -2), (2, (1 << 31) - 1, -2), (3, 0, -2), (4, 255, -2), (8, 255, -2), (8, 264, -2), (8, 240, -2),
        (6, 64, -3), (6, 0, -3), (0, None, -1), (7, None, -1), (9, None, -1), (0, P(FAKE + 1), -4), (7, P(FAKE + 8), -4), (2, 0, 0)])
    t = list(ok)
    t[5], t[4] = 1, 63                                   # transposed: the pitch holds R elements
    assert b.lib().ppo_fp8_quantize(*t) == -2


def test_matmul_refusals(b):
    # A lda sa | B ldb sb block_n | M N K C out ldc ws scratch stream
    ok = [P(FAKE), 256, P(FAKE), P(FAKE), 256, P(FAKE), 128, 4, 100, 256, P(FAKE), b.PPO_BF16, 100, None, None, None]
    _codes(b.lib().ppo_fp8_matmul, ok, [
        (11, 3, -5), (7, -1, -2), (8, 0, -2), (9, 0, -2), (9, 257, -2), (1, 250, -2), (1, 264, -2), (4, 264, -2), (4, 240, -2),
        (12, 99, -2), (14, P(FAKE + 16), -4), (7, (1 << 31) - 1, -2), (6, 64, -3), (0, None, -1), (2, None, -1), (3, None, -1), (5, None, -1),
        (10, None, -1), (0, P(FAKE + 8), -4), (3, P(FAKE + 8), -4), (10, P(FAKE + 1), -4), (7, 0, 0)])


def test_binding_refuses_cpu_tensors(b):
    x = torch.zeros(4, 256)
    with pytest.raises(TypeError):
        b.logprob_topk(x, torch.zeros(4, dtype=torch.int32), 2, 0.7)
    with pytest.raises(TypeError):
        b.logprob_topk_bwd(x, torch.zeros(4), 0.7)
    with pytest.raises(TypeError):
        b.fp8_quantize(x)
    q = torch.zeros(4, 256).to(torch.float8_e4m3fn)
    with pytest.raises(TypeError):
        b.fp8_matmul(q, torch.zeros(2, 4), q, torch.zeros(1, 2))


def test_scratch_is_sized_for_the_operands_device(b, monkeypatch):
    """The plan of a product follows the SMs of the device that runs it, which need not be the current one."""
    current = [0]

    class Guard:
        def __init__(self, at):
            self.at = at

        def __enter__(self):
            self.old, current[0] = current[0], self.at

        def __exit__(self, *_):
            current[0] = self.old

    class Lib:
        @staticmethod
        def ppo_fp8_scratch_bytes(M, N, K):
            return 1000 + current[0]

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(b, "lib", lambda: Lib)
    assert b.fp8_scratch_bytes(600, 2000, 12000) == 1000
    assert b.fp8_scratch_bytes(600, 2000, 12000, torch.device("cuda", 3)) == 1003
    assert b.fp8_scratch_bytes(600, 2000, 12000, "cuda") == 1000 and current == [0]


def test_workspaces_are_cleared_and_read_on_the_stream_of_their_device(b, monkeypatch):
    current, seen = ["cuda:0"], []

    class Guard:
        def __init__(self, at):
            self.at = at

        def __enter__(self):
            self.old, current[0] = current[0], str(self.at)

        def __exit__(self, *_):
            current[0] = self.old

    class Lib:
        @staticmethod
        def ppo_workspace_init(ws, n, stream):
            seen.append((stream, current[0]))
            return 0

        @staticmethod
        def ppo_last_device_status(ws, stream, code):
            seen.append((stream, current[0]))
            return 0

    class Tensor:                                        # stands in for 256 bytes on the second device
        device = torch.device("cuda", 1)
        data_ptr, numel = staticmethod(lambda: 256), staticmethod(lambda: 256)

    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: Tensor)
    monkeypatch.setattr(b, "lib", lambda: Lib)
    monkeypatch.setattr(b, "_ptr", lambda t: t.data_ptr())
    monkeypatch.setattr(b, "_stream", lambda: "stream of " + current[0])
    assert b.last_device_status(b.new_workspace(256, "cuda:1")) == 0
    assert seen == [("stream of cuda:1", "cuda:1")] * 2 and current == ["cuda:0"]
