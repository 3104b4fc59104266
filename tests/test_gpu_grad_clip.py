"""ppo_grad_clip against oracle/sft_oracle.py.

Norm: squares of fp32 values summed eight at a time in fp32 (9 roundings of 2^-24, relative: all are positive), then in fp64: the sum is
off by 9 2^-24, its root by half of that, and rounding the norm adds 2^-24. Results: factor and product are two roundings of 2^-24, then
half a step of the type."""
import numpy as np
import pytest
import torch

from oracle import sft_oracle as O

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


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


def make(sizes, types, seed=0, size=1.0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = torch.empty(n + shift, dtype=types[i % len(types)], device="cuda")[shift:]
        out.append(t.copy_(torch.randn(n, generator=g, device="cuda") * size * (1 + i % 3)))
    return out


def check(P, grads, max_norm, scale=1.0, out=None, **kw):
    want, norm, coef = O.grad_clip([f64(g) for g in grads], max_norm, scale)
    got = P.grad_clip(grads, max_norm, scale=scale, out=out, **kw)
    n, c = [float(x) for x in got]
    e = 4.5 * 2.0 ** -24 + 2.0 ** -23
    if norm < 3e38:
        assert abs(n - norm) <= norm * (e + 2.0 ** -24) + 2.0 ** -149
    assert abs(c - coef) <= coef * (e + 2.0 ** -24)
    for o, w in zip(grads if out is None else out, want):
        # 2^-126: what is smaller loses digits in fp32 itself
        assert (np.abs(f64(o) - w) <= np.abs(w) * 1.01 * (e + 2 * 2.0 ** -24 + HALF[o.dtype]) + 2.0 ** -126).all()
    return norm, coef


LISTS = [[1], [0, 5], [7, 8, 9], [4096, 1, 4096, 4096], [32768, 32769, 65535], [100003, 5, 0, 300000, 17], [13] * 65, [40] * 905 + [70000]]


@pytest.mark.parametrize("sizes", LISTS, ids=[str(len(x)) + "x" + str(sum(x)) for x in LISTS])
@pytest.mark.parametrize("types", [[F32], [BF16], [BF16, F32]])
@pytest.mark.parametrize("max_norm,scale", [(1.0, 1.0), (0.5, -0.25), (1e6, 0.5), (float("inf"), 1.0)])
def test_in_place_and_into_other_tensors(P, sizes, types, max_norm, scale):
    grads = make(sizes, types)
    out = [torch.full_like(g, 3.0, dtype=BF16 if i % 2 else F32) for i, g in enumerate(grads)]
    before = [g.clone() for g in grads]
    check(P, grads, max_norm, scale, out=out)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    check(P, grads, max_norm, scale)


@pytest.mark.parametrize("shift", [1, 3])
def test_tensors_off_alignment_and_neighbours(P, shift):
    flat = torch.full((5000,), 2.0, device="cuda")
    a, b = flat[shift:1000 + shift], flat[2000 + shift:4000]
    check(P, [a, b], 1.0)
    assert (flat[:shift] == 2).all() and (flat[1000 + shift:2000 + shift] == 2).all() and (flat[4000:] == 2).all()
    check(P, make([999, 3], [BF16], shift=shift), 1.0)


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e22, 1e37])
def test_values_whose_squares_leave_fp32(P, size):
    grads = make([5000, 11], [F32], size=size * 0.3)
    norm, coef = check(P, grads, 1.0)
    assert (coef < 1) == (size > 1)
    check(P, make([5000, 11], [BF16, F32], size=size * 0.3, shift=1), 1.0)


def test_mixed_magnitudes_and_zeros(P):
    g = make([100000], [F32])[0]
    g[::2] *= 1e-25
    g[1000:1050] = 0
    check(P, [g, torch.zeros(70000, device="cuda")], 1.0)
    z = [torch.zeros(500, device="cuda"), torch.zeros(3, dtype=BF16, device="cuda")]
    assert P.grad_clip(z, 1.0).tolist() == [0.0, 1.0] and not z[0].any()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 777, 40000])
def test_non_finite_gradients(P, value, at):
    grads = make([40001, 5], [F32, BF16])
    grads[0][at] = value
    ws = P.new_workspace(P.workspace_bytes(1, 1, 8))
    out = [torch.zeros_like(g) for g in grads]
    n = P.grad_clip(grads, 1.0, out=out, workspace=ws)
    assert not torch.isfinite(n).any() and all(torch.isnan(o).all() for o in out) and P.last_device_status(ws) == 32
    P.grad_clip(grads[1:], 1.0, workspace=ws)
    assert P.last_device_status(ws) == 0


def test_same_bits_on_another_stream_and_in_a_graph(P):
    grads = make([70001, 40, 300000], [BF16, F32])
    out = [torch.empty_like(g) for g in grads]
    n = P.grad_clip(grads, 1.0, out=out)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        out2 = [torch.empty_like(g) for g in grads]
        n2 = P.grad_clip(grads, 1.0, out=out2)
    torch.cuda.synchronize()
    assert torch.equal(n, n2) and all(torch.equal(a, b) for a, b in zip(out, out2))
    scratch = torch.empty(P.grad_clip_scratch_bytes(3), dtype=torch.uint8, device="cuda")
    norm = torch.empty(2, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.grad_clip(grads, 1.0, out=out2, scratch=scratch, norm=norm)
    for o in out2:
        o.fill_(7)
    scratch.fill_(255)
    g.replay()
    assert torch.equal(n, norm) and all(torch.equal(a, b) for a, b in zip(out, out2))
    grads[0].mul_(3)
    g.replay()
    assert torch.equal(norm, P.grad_clip(grads, 1.0, out=out)) and all(torch.equal(a, b) for a, b in zip(out, out2))


def test_past_32_bit_offsets(P):
    g = torch.zeros(2 ** 31 + 9, dtype=BF16, device="cuda")
    g[-1], g[5] = 3.0, 4.0
    assert P.grad_clip([g], 2.5).tolist() == [5.0, 0.5]
    assert g[-1] == 1.5 and g[5] == 2


def test_refusals(P):
    g = make([10], [F32])[0]
    with pytest.raises(P.PPOError):
        P.grad_clip([g], 0.0)
    with pytest.raises(P.PPOError):
        P.grad_clip([g], 1.0, scale=0.0)
    with pytest.raises(TypeError):
        P.grad_clip([g[::2]], 1.0)
    with pytest.raises(TypeError):
        P.grad_clip([g.double()], 1.0)
    with pytest.raises(ValueError):
        P.grad_clip([g], 1.0, out=[g[:5]])


def test_a_tensor_is_written_once(P):
    a, b = make([10, 10], [F32])
    empty = a[:0]
    for args in (dict(grads=[a, b, a]), dict(grads=[a, b], out=[a, a])):
        with pytest.raises(ValueError):
            P.grad_clip(max_norm=1.0, **args)
    want = 2 * (f64(a) ** 2).sum()
    out = [torch.empty_like(a), torch.empty_like(a)]
    norm = P.grad_clip([a, a], 1e9, out=out)                    # read twice: allowed
    assert abs(norm[0].item() ** 2 / want - 1) < 16 * 2.0 ** -24 and torch.equal(out[0], out[1])
    P.grad_clip([a, empty, b, empty], 1.0)
