"""ppo_grad_clip at the ends of fp32's range, and lists that name one memory twice."""
import numpy as np
import pytest
import torch

from oracle import sft_oracle as O

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


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


def test_a_result_is_no_other_gradient(P):
    a, b = torch.randn(1000, device="cuda"), torch.randn(1000, device="cuda")
    before = [a.clone(), b.clone()]
    for out in ([b, a], [torch.empty_like(a), a], [b, torch.empty_like(b)]):
        with pytest.raises(ValueError):
            P.grad_clip([a, b], 1.0, out=out)
    flat = torch.randn(3000, device="cuda")
    for grads, out in (([flat[:1000], flat[999:1999]], None), ([flat[:1000]], [flat[1:1001]]), ([a, b], [flat[:1000], flat[500:1500]])):
        with pytest.raises(P.PPOError):
            P.grad_clip(grads, 1.0, out=out)
    assert torch.equal(a, before[0]) and torch.equal(b, before[1])
    want, _, _ = O.grad_clip([f64(a), f64(b)], 1.0, 1.0)
    other = torch.empty_like(b)
    P.grad_clip([a, b], 1.0, out=[a, other])                                         # in place, and beside
    for got, w in ((a, want[0]), (other, want[1])):
        assert (np.abs(f64(got) - w) <= np.abs(w) * 12 * 2.0 ** -24).all()
    assert torch.equal(b, before[1])
    P.grad_clip([flat[:1000], flat[1000:2000], flat[:0]], 1.0)                       # neighbours


@pytest.mark.parametrize("types", [[F32], [BF16], [BF16, F32]])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("max_norm,scale", [(1.0, 1.0), (1e-3, 1.0), (1e-6, -0.5), (1e-30, 1.0), (1e30, 1e-30), (1e30, 3e-42)])
def test_factors_below_fp32(P, types, shift, max_norm, scale):
    """Values near 3e38 whose results are ordinary numbers. Norm and factor as in ordinary lists: 4.5 2^-24 and 2^-23; the product is one rounding
    to fp32, then half a step of the type; what is below 2^-126 loses digits in fp32 itself (half of its last place, 2^-150, here)."""
    sizes = (300000, 70001, 3)
    g = torch.Generator(device="cuda").manual_seed(1)
    grads = [torch.empty(n + shift, dtype=types[i % len(types)], device="cuda")[shift:] for i, n in enumerate(sizes)]
    for t in grads:
        t.copy_((torch.rand(t.numel(), generator=g, device="cuda") * 2 - 1) * 3.2e38)
    grads[1][::3] *= 1e-20
    want, norm, coef = O.grad_clip([f64(t) for t in grads], max_norm, scale)
    out = [torch.full_like(t, 3.0, dtype=BF16 if i % 2 else F32) for i, t in enumerate(grads)]
    n = P.grad_clip(grads, max_norm, scale=scale, out=out)
    P.grad_clip(grads, max_norm, scale=scale)                                       # in place
    e = 4.5 * 2.0 ** -24 + 2.0 ** -23
    for o, w in list(zip(out, want)) + list(zip(grads, want)):
        half = 2.0 ** -8 if o.dtype == BF16 else 2.0 ** -24
        # (the least step is that of the type's subnormal numbers)
        assert (np.abs(f64(o) - w) <= np.abs(w) * 1.01 * (e + 2.0 ** -24 + half) + (2.0 ** -134 if o.dtype == BF16 else 2.0 ** -150) * 1.01).all()
    assert abs(float(n[1]) - coef) <= coef * (e + 2.0 ** -24) + 2.0 ** -150
    assert (float(n[0]) == float("inf")) if norm > 3.41e38 else abs(float(n[0]) - norm) <= norm * (e + 2.0 ** -24) + 2.0 ** -150
