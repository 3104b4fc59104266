"""Arguments of the supervised fine-tuning calls at the ends of their range, and what they refuse before any launch (no GPU)."""
import ctypes as C
import subprocess
import sys

import pytest

FAKE = 0x10000   # a non-null, 256-byte aligned address that is never dereferenced on these paths
P = C.c_void_p


@pytest.fixture(scope="module")
def b():
    from paper_2403_17031_b200 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("M", [1, 2, 3, 100, 9000])
def test_any_number_of_rows_may_be_asked_for_in_a_piece(b, M):
    """More than there are: one piece. (In a process of its own: a division by zero would end this one.)"""
    code = "from paper_2403_17031_b200 import binding as b; print(b.lmhead_xent_scratch_bytes(%d, 64, 1000, %%d))" % M
    most, whole = [subprocess.run([sys.executable, "-c", code % rows], capture_output=True, text=True) for rows in (2 ** 63 - 1, M)]
    assert whole.returncode == 0 and (most.returncode, most.stdout) == (0, whole.stdout)


def test_no_tensor_that_is_clipped_shares_memory_with_another(b):
    """Pass 2 would read what it has scaled already, or not yet. (Refused before the device is looked for; what is not refused does not get past
    that here, so these calls name a device's error or, on one, are not made.)"""
    import torch
    I64, I32, PTR = C.c_int64, C.c_int32, C.c_void_p

    def call(ins, numel, types, outs=None, out_types=None):
        n = len(ins)
        arr = lambda t, x: None if x is None else (t * n)(*x)                       # noqa: E731
        return b.lib().ppo_grad_clip(n, arr(PTR, ins), arr(I64, numel), arr(I32, types), arr(PTR, outs), arr(I32, out_types), 1.0, 1.0,
                                     P(FAKE), None, P(FAKE), None)

    A, B, X, Y = [i << 24 for i in (1, 2, 3, 4)]
    F, H = b.PPO_F32, b.PPO_BF16
    refused = [
        ([A, B], [8, 8], [F, F], [B, A], [F, F]),                    # swapped
        ([A, B], [8, 8], [F, F], [X, A], [F, F]),                    # one into the other's place
        ([A, A + 16], [8, 8], [F, F]),                               # parts in place
        ([A, A], [8, 8], [F, F]),
        ([A, A], [8, 8], [F, F], [A, X], [F, F]),                    # read by one, scaled in place by the other
        ([A, B], [8, 8], [H, H], [X, X + 28], [F, F]),               # fp32 results of bf16: 32 bytes each
        ([A], [8], [H], [A + 2], [H]),                               # a step further
        ([A], [8], [F], [A + 16], [H]),
        ([A] + [B + 64 * i for i in range(300)], [8] + [16] * 300, [F] * 301, [X] + [Y + 64 * i for i in range(299)] + [X + 28], [F] * 301),
    ]
    for args in refused:
        assert call(*args) == -3, args
    if torch.cuda.is_available():
        return
    for args in [([A, A + 32], [8, 8], [F, F]), ([A, A], [8, 8], [F, F], [X, Y], [F, F]),          # read twice
                 ([A, B], [8, 8], [F, F], [A, Y], [F, F]), ([A, A], [8, 0], [F, F]), ([A, B], [8, 8], [H, H], [X, X + 32], [F, F]),
                 ([A + 64 * i for i in range(300)][::-1], [16] * 300, [F] * 300)]:
        assert call(*args) > 0, args


def test_addresses_that_numbers_cannot_have(b):
    """Every pointer whose misalignment would fault is refused: results, the divisor, and a workspace that ppo_workspace_init cannot have made."""
    # H ldh W ldw layout M K V | labels mask ignore temperature scale denom piece | loss nll lse dH lddh dW lddw | ws scratch stream
    ok = [P(FAKE), 256, P(FAKE), 1000, 0, 4, 256, 1000, P(FAKE), None, -100, 1.0, 1.0, None, 0, P(FAKE), P(FAKE), None, P(FAKE), 256,
          P(FAKE), 1000, None, P(FAKE), None]
    embed = [P(FAKE), b.PPO_BF16, 1000, 64, 64, P(FAKE), 4, 1.0, P(FAKE), b.PPO_F32, 64, None, None]
    bwd = [P(FAKE), b.PPO_BF16, 4, 64, 64, P(FAKE), 1000, 1.0, -1, P(2 * FAKE), b.PPO_F32, 64, 0, None, P(FAKE), None]
    one = lambda t, x: (t * 1)(x)                                                   # noqa: E731
    clip = [1, one(C.c_void_p, FAKE), one(C.c_int64, 8), one(C.c_int32, 0), None, None, 1.0, 1.0, P(FAKE), None, P(FAKE), None]
    for name, args, at in (("ppo_lmhead_xent", ok, ((13, 2), (15, 2), (16, 1), (17, 3), (22, 64))), ("ppo_embed", embed, ((11, 128),)),
                           ("ppo_embed_bwd", bwd, ((13, 8),)), ("ppo_grad_clip", clip, ((8, 2), (9, 4)))):
        for i, off in at:
            bad = list(args)
            bad[i] = P(FAKE + off)
            assert getattr(b.lib(), name)(*bad) == -4, (name, i)
