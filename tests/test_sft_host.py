"""Refusals of the supervised fine-tuning calls: the documented codes, before any launch (no GPU)."""
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


def test_xent_refusals(b):
    # H ldh W ldw layout M K V | labels mask ignore temperature scale denom piece | loss nll lse dH lddh dW lddw | ws scratch stream
    ok = [P(FAKE), 256, P(FAKE), 1000, 0, 4, 256, 1000, P(FAKE), None, -100, 1.0, 1.0, None, 0, P(FAKE), P(FAKE), None, P(FAKE), 256,
          P(FAKE), 1000, None, P(FAKE), None]
    _codes(b.lib().ppo_lmhead_xent, ok, [
        (4, 2, -3), (5, -1, -2), (5, 1 << 31, -2), (6, 0, -2), (7, 0, -2), (7, 1 << 31, -2), (14, -1, -2), (1, 255, -2), (3, 999, -2),
        (19, 255, -2), (21, 999, -2), (11, 0.0, -3), (11, float("nan"), -3), (12, float("inf"), -3), (0, None, -1), (2, None, -1),
        (8, None, -1), (15, None, -1), (16, None, -1), (23, None, -1), (1, 257, -6), (3, 1001, -6), (0, P(FAKE + 8), -4),
        (2, P(FAKE + 8), -4), (23, P(FAKE + 16), -4), (18, P(FAKE + 1), -4), (20, P(FAKE + 1), -4), (8, P(FAKE + 2), -4)])
    vk = list(ok)
    vk[4] = 1                                            # stored [V, K]: the pitch holds K elements
    vk[3] = 255
    assert b.lib().ppo_lmhead_xent(*vk) == -2
    n = b.lmhead_xent_scratch_bytes
    assert n(0, 256, 1000) == 0 and n(4, 256, 0) == 0
    # the piece bounds the scratch: 256 rows x V in 16 bits, the sums of dW (whole tiles), what is per row of M, and two tiles a pair of blocks
    assert n(1 << 16, 64, 50304, 256) < 2 * 256 * 50304 + 4 * 512 * 50688 + (1 << 16) * (128 + 12) + 256 * (394 * 16 + 256) + (84 << 20)
    assert n(4, 256, 1000, 0, False, False) < n(4, 256, 1000, 0, True, False) < n(4, 256, 1000)


def test_embed_refusals(b):
    # table dtype V K lde | tokens N scale | out dtype ldo ws stream
    ok = [P(FAKE), b.PPO_BF16, 1000, 64, 64, P(FAKE), 4, 1.0, P(FAKE), b.PPO_F32, 64, None, None]
    _codes(b.lib().ppo_embed, ok, [
        (1, 2, -5), (9, 7, -5), (2, 0, -2), (3, 0, -2), (4, 63, -2), (6, -1, -2), (6, 1 << 31, -2), (10, 63, -2), (7, float("nan"), -3),
        (0, None, -1), (5, None, -1), (8, None, -1), (0, P(FAKE + 1), -4), (8, P(FAKE + 2), -4), (5, P(FAKE + 2), -4), (6, 0, 0)])


def test_embed_bwd_refusals(b):
    # dY dtype N K ldy tokens V | scale padding | dE dtype lde accumulate | ws scratch stream
    ok = [P(FAKE), b.PPO_BF16, 4, 64, 64, P(FAKE), 1000, 1.0, -1, P(2 * FAKE), b.PPO_F32, 64, 0, None, P(FAKE), None]
    _codes(b.lib().ppo_embed_bwd, ok, [
        (1, 2, -5), (10, 7, -5), (2, -1, -2), (2, 1 << 31, -2), (3, 0, -2), (4, 63, -2), (6, 0, -2), (11, 63, -2),
        (7, float("inf"), -3), (0, None, -1), (5, None, -1), (9, None, -1), (14, None, -1), (0, P(FAKE + 1), -4),
        (9, P(FAKE + 2), -4), (14, P(FAKE + 16), -4)])
    none = list(ok)
    none[2], none[12] = 0, 1                             # nothing to add
    assert b.lib().ppo_embed_bwd(*none) == 0
    assert b.embed_bwd_scratch_bytes(0, 64, 1000) == 0 and b.embed_bwd_scratch_bytes(1, 64, 1000) > 0


def test_grad_clip_refusals(b):
    ins = (C.c_void_p * 2)(FAKE, 2 * FAKE)
    outs = (C.c_void_p * 2)(FAKE, 3 * FAKE)
    numel, bad = (C.c_int64 * 2)(8, 8), (C.c_int64 * 2)(8, -1)
    f32, mixed, wrong = (C.c_int32 * 2)(0, 0), (C.c_int32 * 2)(1, 0), (C.c_int32 * 2)(0, 2)
    # n in numel dtype out dtype scale max_norm norm ws scratch stream
    ok = [2, ins, numel, f32, outs, f32, 1.0, 1.0, P(FAKE), None, P(FAKE), None]
    _codes(b.lib().ppo_grad_clip, ok, [
        (0, 0, -2), (0, -1, -2), (2, bad, -2), (6, 0.0, -3), (6, float("nan"), -3), (7, 0.0, -3), (7, float("nan"), -3), (7, -1.0, -3),
        (1, None, -1), (2, None, -1), (3, None, -1), (5, None, -1), (8, None, -1), (10, None, -1), (3, wrong, -5), (5, wrong, -5),
        (1, (C.c_void_p * 2)(FAKE, None), -1), (4, (C.c_void_p * 2)(FAKE, None), -1), (1, (C.c_void_p * 2)(FAKE, FAKE + 2), -4),
        (10, P(FAKE + 16), -4), (5, mixed, -3)])         # the last: in place, in another type
    assert b.grad_clip_scratch_bytes(0) == 0


def test_binding_refuses_what_does_not_fit(b):
    x, t = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        b.embed(x, t)
    with pytest.raises(TypeError):
        b.embed_bwd(x, t, 10)
    with pytest.raises(TypeError):
        b.lmhead_xent(x.bfloat16(), torch.zeros(64, 32, dtype=torch.bfloat16), t)
    with pytest.raises(TypeError):
        b.grad_clip([x], 1.0)
    with pytest.raises(ValueError):
        b.grad_clip([], 1.0)


@pytest.mark.parametrize("K,V", [(1, 5), (5, 1), (1, 1), (3, 4), (1, 8), (8, 1)])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("more", [0, 3])
def test_a_gradient_lies_as_its_weight_says_also_with_a_size_of_one(b, K, V, layout, more):
    """Strides of a size of one say nothing: address of (k, v) as the library forms it, against torch's."""
    bf16 = torch.bfloat16
    rows, inner = (K, V) if layout == b.W_KV else (V, K)
    for t in (torch.empty(rows, inner + more, dtype=bf16)[:, :inner], torch.empty(rows, inner, dtype=bf16),
              torch.empty(inner, rows, dtype=bf16).t(), torch.empty(rows, 2 * inner, dtype=bf16)[:, ::2]):
        dW = t if layout == b.W_KV else t.t()
        assert dW.shape == (K, V)
        fits = all(k * dW.stride(0) + v * dW.stride(1) == (k * (dW.stride(0) if layout == b.W_KV else 1) + v * (1 if layout == b.W_KV else dW.stride(1)))
                   for k in range(K) for v in range(V)) and (rows <= 1 or t.stride(0) >= inner)
        if not fits:
            with pytest.raises(ValueError):
                b._head_gradient(dW, layout, -1, "dW")
            continue
        at, pitch = b._head_gradient(dW, layout, -1, "dW")
        assert at == dW.data_ptr() and pitch >= inner
        for k in range(K):
            for v in range(V):
                r, i = (k, v) if layout == b.W_KV else (v, k)
                assert r * pitch + i == k * dW.stride(0) + v * dW.stride(1)
