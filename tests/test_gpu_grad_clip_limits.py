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
