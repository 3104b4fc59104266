"""ppo_embed and ppo_embed_bwd against oracle/sft_oracle.py.

Forward: one product, rounded to fp32 and then to the result's type: half a step of each. Gradient: n summands in fp32, each addition off by at most
2^-24 of its partial sum (the products with 1 are exact), the scale one more, an fp32 sum that is added to one more, then half a step of the type."""
import numpy as np
import pytest
import torch

from oracle import sft_oracle as O
from parity import npy

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


def f64(t):
    return t.detach().double().cpu().numpy()


def rows(R, C, dtype, pad=0, seed=0, shift=0):
    """[R, C] at a row pitch of C + pad, `shift` elements off the start of its memory."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.full((R * (C + pad) + shift,), 9.0, dtype=dtype, device="cuda")[shift:]
    x = flat.view(R, C + pad)[:, :C]
    x.copy_(torch.randn(R, C, generator=g))
    return x


def text(N, V, seed=0):
    """Ids of which a few make up most."""
    g = torch.Generator().manual_seed(seed)
    return (torch.rand(N, generator=g) ** 6 * V).to(I32).clamp(max=V - 1).cuda()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("N,K,V,pad", [(1, 1, 1, 0), (53, 256, 1000, 0), (5, 4096, 70, 8), (700, 33, 50, 0), (5000, 64, 300, 3), (4999, 1021, 100, 0)])
def test_lookup(P, dtype, out, N, K, V, pad):
    E, tokens = rows(V, K, dtype, pad), text(N, V)
    y = P.embed(E, tokens, scale=1.7, out_dtype=out)
    want = O.embed(f64(E), npy(tokens), 1.7)
    assert (np.abs(f64(y) - want) <= (HALF[out] + 2.0 ** -24) * (1 + 2.0 ** -8) * np.abs(want)).all()
    assert torch.equal(P.embed(E, tokens).float(), E[tokens.long()].float())


def test_lookup_shapes_bad_tokens_and_pitches(P):
    E = rows(40, 24, BF16)
    tokens = text(6, 40).view(2, 3)
    assert P.embed(E, tokens).shape == (2, 3, 24)
    tokens[0, 1], tokens[1, 2] = 40, -1
    ws = P.new_workspace(P.workspace_bytes(6, 1, 40))
    buf = torch.full((6, 30), 5.0, dtype=F32, device="cuda")
    y = P.embed(E, tokens, out=buf[:, :24], workspace=ws)
    bad = torch.tensor([False, True, False, False, False, True], device="cuda")
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], E[tokens.view(-1)[~bad].long()].float()) and (buf[:, 24:] == 5).all()
    assert P.last_device_status(ws) == 1
    assert P.embed(E, tokens[:0]).shape == (0, 3, 24)


def check_bwd(P, dY, tokens, V, scale=1.0, padding_id=-1, out=None, base=None, **kw):
    N, K = dY.shape
    o = P.embed_bwd(dY, tokens, V, scale=scale, padding_id=padding_id, out=out, accumulate=base is not None, **kw)
    b = None if base is None else f64(base)
    want, size = O.embed_bwd(f64(dY), npy(tokens), V, scale, padding_id, b)
    count = np.bincount(np.clip(npy(tokens), 0, V - 1), minlength=V)[:, None]
    tol = (count + 2) * 2.0 ** -24 * (size + (0 if b is None else np.abs(b))) + HALF[o.dtype] * np.abs(want)
    assert (np.abs(f64(o) - want) <= 1.01 * tol).all()
    return o


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("N,K,V,pad", [(1, 1, 1, 0), (1, 64, 300, 0), (53, 256, 1000, 0), (700, 33, 50, 0), (3000, 72, 20, 8), (4999, 1021, 100, 3),
                                       (8192, 16, 5000, 0), (8193, 24, 5000, 0), (20000, 40, 300, 0), (70001, 8, 70000, 0)])
def test_gradient(P, dtype, out, N, K, V, pad):
    check_bwd(P, rows(N, K, dtype, pad), text(N, V), V, scale=0.5, out_dtype=out)


@pytest.mark.parametrize("N", [1, 40, 700, 9000])
def test_gradient_of_one_token_of_distinct_tokens_and_of_none(P, N):
    dY = rows(N, 48, F32)
    check_bwd(P, dY, torch.full((N,), 7, dtype=I32, device="cuda"), 9)
    perm = torch.randperm(N, generator=torch.Generator().manual_seed(1)).to(I32).cuda()
    d = P.embed_bwd(dY, perm, N)
    assert torch.equal(d[perm.long()], dY)
    d = P.embed_bwd(dY, torch.full((N,), 3, dtype=I32, device="cuda"), 9, padding_id=3)
    assert not d.any()


@pytest.mark.parametrize("N", [300, 9000])
def test_padding_bad_tokens_and_canaries(P, N):
    dY, tokens = rows(N, 56, BF16, pad=8), text(N, 120)
    tokens[::7] = 1
    ws = P.new_workspace(P.workspace_bytes(N, 1, 120))
    buf = torch.full((121, 60), 5.0, dtype=F32, device="cuda")
    d = check_bwd(P, dY, tokens, 120, padding_id=1, out=buf[:120, :56], workspace=ws)
    assert not d[1].any() and (buf[:, 56:] == 5).all() and (buf[120] == 5).all() and P.last_device_status(ws) == 0
    tokens[5], tokens[N - 1], tokens[8] = 120, -1, -(2 ** 31)
    check_bwd(P, dY, tokens, 120, padding_id=1, workspace=ws)
    assert P.last_device_status(ws) == 1


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("N", [40, 2000, 9000])
def test_accumulating_leaves_other_rows_alone(P, out, N):
    dY, tokens = rows(N, 72, BF16), text(N, 3000)
    base = rows(3000, 72, out, seed=5)
    seen = torch.zeros(3000, dtype=torch.bool, device="cuda")
    seen[tokens.long()] = True
    base[~seen] = torch.nan
    before = base.clone()
    clean = before.nan_to_num()
    o = P.embed_bwd(dY, tokens, 3000, out=base, accumulate=True)
    assert torch.isnan(o[~seen]).all() and torch.isfinite(o[seen]).all()
    again = clean.clone()
    check_bwd(P, dY, tokens, 3000, out=again, base=clean)
    assert torch.equal(again[seen], o[seen])
    assert P.embed_bwd(dY[:0], tokens[:0], 3000, out=again, accumulate=True) is again
    assert not P.embed_bwd(dY[:0], tokens[:0], 3000, out=again).any()


@pytest.mark.parametrize("N", [50, 5000, 20000])
def test_same_bits_on_another_stream_and_in_a_graph(P, N):
    V = 2000
    dY, tokens = rows(N, 40, BF16), text(N, V)
    one = P.embed_bwd(dY, tokens, V, padding_id=0)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        a = P.embed_bwd(dY, tokens, V, padding_id=0)
        y = P.embed(one, tokens)
    torch.cuda.synchronize()
    assert torch.equal(a, one) and torch.equal(y, one[tokens.long()])
    scratch = torch.full((P.embed_bwd_scratch_bytes(N, 40, V),), 255, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = P.embed_bwd(dY, tokens, V, padding_id=0, scratch=scratch)
    scratch.fill_(255)
    g.replay()
    assert torch.equal(o, one)
    tokens.copy_(text(N, V, seed=9))
    g.replay()
    assert torch.equal(o, P.embed_bwd(dY, tokens, V, padding_id=0))


def test_rows_off_alignment(P):
    dY, E, tokens = rows(90, 64, BF16, shift=3), rows(50, 64, BF16, shift=1), text(90, 50)
    check_bwd(P, dY, tokens, 50)
    assert torch.equal(P.embed(E, tokens), E[tokens.long()])


def test_past_32_bit_offsets(P):
    """A table of 2^31 elements and more: the last rows' gradient and lookup."""
    V, K = 70000, 32768
    E = torch.empty((V, K), dtype=BF16, device="cuda")
    E[-3:] = rows(3, K, BF16)
    tokens = torch.tensor([V - 1, V - 3, V - 1], dtype=I32, device="cuda")
    y = P.embed(E, tokens)
    assert torch.equal(y, E[tokens.long()])
    d = P.embed_bwd(y, tokens, V, out=E)
    assert torch.equal(d[V - 1], (y[0].float() + y[2].float()).to(BF16)) and torch.equal(d[V - 3], y[1])
    assert not d[V - 2].any() and not d[: V - 3].any()


def test_refusals(P):
    E, tokens = rows(50, 64, BF16), text(9, 50)
    with pytest.raises(TypeError):
        P.embed(E, tokens.long())
    with pytest.raises(TypeError):
        P.embed(E.to(torch.float16), tokens)
    with pytest.raises(ValueError):
        P.embed_bwd(rows(9, 64, F32), tokens[:8], 50)
    with pytest.raises(ValueError):
        P.embed_bwd(rows(9, 64, F32), tokens, 50, accumulate=True)
    with pytest.raises(ValueError):
        P.embed_bwd(rows(9, 64, F32), tokens, 50, out=rows(49, 64, F32))
