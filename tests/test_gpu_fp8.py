"""ppo_fp8_quantize and ppo_fp8_matmul against oracle/fp8_oracle.py.

Quantisation: the definition names its fp32 operations, so scales and values are exact. Product: each output may be off by half a step
of its type, relative, and by gamma times the sum of the absolute products: products of two e4m3 values are exact in fp32; a block's 128
of them and the sum over the blocks are fp32 additions, each off by at most 2^-23 of its (absolute) partial sum whether it rounds or cuts
off, and the factors add three roundings per block: gamma = (128 + blocks + 3) * 2^-23."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as O
from parity import npy

pytestmark = pytest.mark.gpu
F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


def _matrix(R, C, dtype, pad=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.zeros(R, C + pad, dtype=dtype, device="cuda")[:, :C]
    x.copy_((torch.randn(R, C, generator=g) * torch.exp(torch.randn(R, 1, generator=g))).to(dtype))
    return x


def _check_quantize(P, x, block, transpose):
    y = (x.t() if transpose else x).float().cpu().numpy()
    q, s = P.fp8_quantize(x, block, transpose)
    wq, wsc = O.quantize(y, block)
    assert tuple(q.shape) == y.shape and q.dtype == F8 and q.stride(0) % 16 == 0
    assert np.array_equal(npy(s), wsc, equal_nan=True)
    assert np.array_equal(npy(q.float()).astype(np.float64), wq, equal_nan=True)
    return q, s


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("R,C,pad", [(1, 1, 0), (1, 128, 0), (128, 1, 0), (300, 577, 0), (33, 1000, 3), (130, 4096, 8), (257, 255, 1)])
def test_quantize_matches_oracle(P, dtype, block, transpose, R, C, pad):
    _check_quantize(P, _matrix(R, C, dtype, pad), block, transpose)


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_zero_tiny_huge_and_non_finite_blocks(P, block, transpose):
    x = _matrix(400, 520, F32)
    x[:140, :140] = 0
    x[150:290, 150:290] *= 1e-35                              # below the smallest block maximum that is scaled exactly
    x[300:, 300:420] *= 1e37
    x[10, 500] = torch.nan
    x[390, 10] = -torch.inf
    _check_quantize(P, x, block, transpose)


def test_quantize_leaves_bytes_behind_the_rows_alone(P):
    x = _matrix(70, 200, BF16)
    buf = torch.full((70, 224), 3.0, device="cuda").to(F8)
    s = torch.empty(2, 70, device="cuda")
    P.fp8_quantize(x, 1, out=(buf[:, :200], s))
    assert (buf[:, 200:].float() == 3.0).all()
    with pytest.raises(ValueError):
        P.fp8_quantize(x, 128, out=(buf[:, :200], s))
    with pytest.raises(TypeError):
        P.fp8_quantize(x, 1, out=(buf[:, :200].float(), s))
    with pytest.raises(P.PPOError):
        P.fp8_quantize(x, 64)
    assert P.fp8_quantize(x[:0])[0].shape == (0, 200)


def _operands(P, M, N, K, block_n, seed=0):
    a, sa = P.fp8_quantize(_matrix(M, K, BF16, seed=seed), 1)
    b, sb = P.fp8_quantize(_matrix(N, K, BF16, seed=seed + 1), block_n)
    return a, sa, b, sb


def _check_matmul(P, M, N, K, block_n, out_dtype, ops=None, out=None):
    a, sa, b, sb = ops or _operands(P, M, N, K, block_n)
    ws = P.new_workspace(256)
    c = P.fp8_matmul(a, sa, b, sb, block_n, out_dtype, workspace=ws, out=out)
    assert P.last_device_status(ws) == 0
    w, size = O.matmul(npy(a.float()), npy(sa), npy(b.float()), npy(sb), block_n)
    got = c.double().cpu().numpy()
    gamma = (128 + -(-K // 128) + 3) * 2.0 ** -23
    assert np.isfinite(got).all()
    err = np.abs(got - w) - torch.finfo(out_dtype).eps / 2 * np.abs(w) - gamma * size
    assert (err <= 0).all(), (np.abs(got - w).max(), int((err > 0).sum()))
    return c


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K,block_n", [
    (1, 1, 1, 128), (1, 300, 128, 128), (1, 1000, 577, 1), (7, 129, 4096, 128), (16, 256, 1000, 1), (17, 255, 640, 128),
    (64, 1024, 512, 128), (65, 333, 333, 1), (128, 128, 128, 128), (129, 257, 130, 128), (300, 1000, 577, 128), (300, 1000, 577, 1),
    (513, 640, 1152, 128), (1000, 1100, 260, 1), (5000, 8, 300, 128), (1500, 1500, 5, 1), (53, 512, 20000, 128), (700, 2000, 1024, 128)])
def test_matmul_matches_oracle(P, out_dtype, M, N, K, block_n):
    _check_matmul(P, M, N, K, block_n, out_dtype)


@pytest.mark.parametrize("out_dtype,block_n", [(F32, 128), (BF16, 1)])
@pytest.mark.parametrize("M,N,K", [(600, 2000, 12000), (257, 15000, 15400), (2600, 4100, 13200)])
def test_matmul_with_tiles_cut_along_k(P, M, N, K, out_dtype, block_n):
    """Sizes whose last round of tiles is shared by all pairs of SMs: with scratch and without, and bit for bit twice."""
    assert P.fp8_scratch_bytes(M, N, K) > 0
    a, sa, b, sb = _operands(P, M, N, K, block_n)
    got = P.fp8_matmul(a, sa, b, sb, block_n, out_dtype)
    scratch = torch.empty(P.fp8_scratch_bytes(M, N, K), dtype=torch.uint8, device="cuda").fill_(255)
    out = torch.full((M, N + 1), 3.0, dtype=out_dtype, device="cuda")
    again = P.fp8_matmul(a, sa, b, sb, block_n, out_dtype, out=out[:, :N], scratch=scratch)     # (rows at odd addresses)
    assert torch.equal(got, again) and (out[:, N:] == 3.0).all()
    cols = torch.cat([torch.arange(0, 130), torch.arange(N - 140, N)])
    w, size = O.matmul(npy(a.float()), npy(sa), npy(b.float())[cols], npy(sb)[:, cols] if block_n == 1 else
                       np.repeat(npy(sb), 128, axis=0)[cols].T.copy(), 1)
    gamma = (128 + -(-K // 128) + 3) * 2.0 ** -23
    err = np.abs(got[:, cols.cuda()].double().cpu().numpy() - w) - torch.finfo(out_dtype).eps / 2 * np.abs(w) - gamma * size
    assert (err <= 0).all(), int((err > 0).sum())
    with pytest.raises(ValueError):
        P.fp8_matmul(a, sa, b, sb, block_n, out_dtype, scratch=scratch[256:])


def test_matmul_results_do_not_depend_on_bytes_behind_k_or_on_the_pitch(P):
    M, N, K = 150, 260, 200
    a, sa, b, sb = _operands(P, M, N, K, 128)
    want = _check_matmul(P, M, N, K, 128, F32, (a, sa, b, sb))
    wide = lambda t: torch.cat([t.float(), torch.full((t.shape[0], 56), torch.nan, device="cuda")], 1).to(F8)[:, :K]   # noqa: E731
    got = P.fp8_matmul(wide(a), sa, wide(b), sb, out_dtype=F32)
    assert torch.equal(got, want)
    buf = torch.full((M, N + 3), 5.0, device="cuda")
    P.fp8_matmul(a, sa, b, sb, out=buf[:, :N])
    assert torch.equal(buf[:, :N], want) and (buf[:, N:] == 5.0).all()


@pytest.mark.parametrize("M,N,pad", [(20, 300, 4), (700, 2000, 8), (700, 2000, 3)])
def test_matmul_leaves_what_lies_behind_its_rows_and_columns_alone(P, M, N, pad):
    a, sa, b, sb = _operands(P, M, N, 640, 128)
    for dtype in (BF16, F32):
        want = P.fp8_matmul(a, sa, b, sb, out_dtype=dtype)
        buf = torch.full((M + 5, N + pad), 5.0, dtype=dtype, device="cuda")
        P.fp8_matmul(a, sa, b, sb, out=buf[:M, :N])
        assert torch.equal(buf[:M, :N], want) and (buf[M:] == 5.0).all() and (buf[:, N:] == 5.0).all()


def test_offsets_past_32_bits(P):
    """A matrix of 2.3e9 elements, and a product of as many: the last rows and columns are those of a small call."""
    M, N = 45056, 50304
    x = torch.zeros(M, N, dtype=BF16, device="cuda")
    x[-130:] = _matrix(130, N, BF16)
    q, s = P.fp8_quantize(x, 1)
    wq, wsc = P.fp8_quantize(x[-130:], 1)
    assert torch.equal(q[-130:].float(), wq.float()) and torch.equal(s[:, -130:], wsc) and not q[:1000].float().any()
    del x, q
    a, sa, b, sb = _operands(P, M, N, 128, 128)
    c = P.fp8_matmul(a, sa, b, sb)
    tail = P.fp8_matmul(a[-300:], sa[:, -300:].contiguous(), b, sb)
    assert torch.equal(c[-300:], tail)


@pytest.mark.parametrize("M", [1, 40, 400])
def test_matmul_nan_stays_in_its_row_and_column(P, M):
    N, K = 300, 512
    x, y = _matrix(M, K, BF16), _matrix(N, K, BF16, seed=1)
    x[M // 2, 5] = torch.nan
    a, sa = P.fp8_quantize(x, 1)
    b, sb = P.fp8_quantize(y, 128)
    c = P.fp8_matmul(a, sa, b, sb)
    nan = torch.isnan(c)
    assert nan[M // 2].all() and int(nan.sum()) == N


def test_matmul_refusals(P):
    a, sa, b, sb = _operands(P, 20, 40, 256, 128)
    with pytest.raises(ValueError):
        P.fp8_matmul(a, sa, b[:, :128], sb)
    with pytest.raises(ValueError):
        P.fp8_matmul(a, sa, b, sb, block_n=1)
    with pytest.raises(ValueError):
        P.fp8_matmul(a, sa[:, :19], b, sb)
    with pytest.raises(TypeError):
        P.fp8_matmul(a.float(), sa, b, sb)
    with pytest.raises(TypeError):
        P.fp8_matmul(a, sa.t().contiguous().t(), b, sb)
    with pytest.raises(TypeError):
        P.fp8_matmul(a, sa, b, sb, out_dtype=torch.float16)
    odd = torch.zeros(20, 250, device="cuda").to(F8)
    with pytest.raises(P.PPOError):
        P.fp8_matmul(odd, sa, odd, torch.zeros(1, 2, device="cuda"))   # a pitch that is not a multiple of 16
    assert P.fp8_matmul(a[:0], sa[:, :0].contiguous(), b, sb).shape == (0, 40)


@pytest.mark.parametrize("M", [3, 200, 1500])
def test_matmul_on_another_stream_in_a_graph_and_bit_for_bit(P, M):
    N, K = 2000, 1024
    a, sa, b, sb = _operands(P, M, N, K, 128)
    want = P.fp8_matmul(a, sa, b, sb, out_dtype=F32)
    out = torch.zeros_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        P.fp8_matmul(a, sa, b, sb, out=out)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.fp8_matmul(a, sa, b, sb, out=out)
    for _ in range(5):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)


def test_a_chain_from_hidden_states_to_their_gradient(P):
    """8-bit LM head: logits, scores and alternatives, their gradient, and the gradient on the hidden states, each stage against
    its definition on the stage before."""
    from oracle import topk_oracle as T
    M, K, V, k = 70, 512, 3000, 10
    h = (_matrix(M, K, BF16) * 0.3).contiguous()
    w = (_matrix(K, V, BF16, seed=2) * 0.05).contiguous()
    hq, hs = P.fp8_quantize(h, 1)
    wq, wsc = P.fp8_quantize(w, 128, transpose=True)          # [V, K], for the logits
    logits = _check_matmul(P, M, V, K, 128, BF16, (hq, hs, wq, wsc))
    tok = torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(4), dtype=torch.int32).cuda()
    f = P.logprob_topk(logits, tok, k, 0.7)
    o = T.topk(logits.double().cpu().numpy(), npy(tok)[:, None], k, np.float32(0.7))
    assert np.array_equal(npy(f["top_ids"]), o["top_ids"]) and np.abs(npy(f["top_logprob"]) - o["top_logprob"]).max() < 1e-4
    g = torch.full((M, 1), -1.0 / M, device="cuda")
    d = P.logprob_topk_bwd(logits, f["lse"], 0.7, tokens=tok, dlogprob=g)["dlogits"]
    old = P.logprob_bwd(logits, tok, torch.ones(M, dtype=torch.uint8, device="cuda"), g.view(M), 0.7,
                        P.new_workspace(P.workspace_bytes(M, 1, V)))["dlogits"]
    assert (d.float() - old.float()).abs().max() <= 2.0 ** -8 * old.float().abs().max()
    dq, ds = P.fp8_quantize(d, 1)
    w2, w2s = P.fp8_quantize(w, 128)                          # [K, V], for the gradient
    assert torch.equal(w2.float(), wq.float().t()) and torch.equal(w2s, wsc.t())
    _check_matmul(P, M, K, V, 128, F32, (dq, ds, w2, w2s))


@pytest.mark.parametrize("out_dtype,block_n", [(F32, 128), (BF16, 1)])
@pytest.mark.parametrize("M,N,K", [(5, 40000, 1100), (16, 37889, 385), (32, 38017, 700), (17, 40001, 129), (20, 50304, 1024)])
def test_matmul_of_few_rows_with_a_long_weight(P, M, N, K, out_dtype, block_n):
    """(more tiles of 128 weight rows than two for each SM)"""
    _check_matmul(P, M, N, K, block_n, out_dtype)


@pytest.mark.parametrize("M,N,K", [(600, 2000, 12000), (257, 15000, 15400)])
def test_tiles_cut_along_k_on_another_stream_in_graphs_and_two_at_a_time(P, M, N, K):
    """The sums and their join (a dependent launch), with scratch of the caller's and scratch allocated inside the call."""
    a, sa, b, sb = _operands(P, M, N, K, 128)
    a2, sa2 = P.fp8_quantize(_matrix(M, K, BF16, seed=5), 1)
    need = P.fp8_scratch_bytes(M, N, K)
    assert need > 0
    wants = [P.fp8_matmul(a, sa, b, sb, out_dtype=F32), P.fp8_matmul(a2, sa2, b, sb, out_dtype=F32)]
    assert not torch.equal(*wants)
    outs = [torch.zeros_like(w) for w in wants]
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(255)
    calls = [lambda: P.fp8_matmul(a, sa, b, sb, out=outs[0], scratch=scratch), lambda: P.fp8_matmul(a2, sa2, b, sb, out=outs[1])]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s, call in zip(streams, calls):
        with torch.cuda.stream(s):
            call()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, wants))
    graphs = []
    for s, call in zip(streams, calls):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            call()
            call()                                              # (the second call's kernels follow the first one's join)
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, wants))


@pytest.mark.parametrize("dtype,N,pad", [(F32, 2045, 3), (F32, 2046, 2), (F32, 2047, 1), (F32, 1985, 31), (BF16, 2041, 7), (BF16, 2044, 4),
                                         (BF16, 2047, 1), (BF16, 1985, 63), (BF16, 1983, 1), (F32, 257, 3), (BF16, 257, 7)])
@pytest.mark.parametrize("M,K", [(700, 640), (2000, 300), (600, 12000)])
def test_matmul_leaves_columns_behind_an_odd_edge_alone(P, M, K, dtype, N, pad):
    """Rows of C at a pitch of 16 bytes that end inside 16 bytes."""
    a, sa, b, sb = _operands(P, M, N, K, 128)
    want = P.fp8_matmul(a, sa, b, sb, out_dtype=F32)
    buf = torch.full((M, N + pad), 5.0, dtype=dtype, device="cuda")
    P.fp8_matmul(a, sa, b, sb, out=buf[:, :N])
    assert torch.equal(buf[:, :N], want.to(dtype)) and (buf[:, N:] == 5.0).all()
