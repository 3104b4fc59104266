"""pipeline.Fp8LMHead: hidden states to scores and back, against the definitions in fp64 on the quantised operands.

Logits and gradients are bf16: half a step, 2^-8 relative. The fp64 reference takes the kernel's own bf16 logits for everything behind
them, so that each stage is compared with its definition."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as F
from oracle import topk_oracle as T
from parity import TOL_LOGPROB, npy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


def _setup(M, K, V, n, k, seed=0):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn(K, V, generator=g) * 0.1).to(torch.bfloat16).cuda()
    H = torch.randn(M, K, generator=g).to(torch.bfloat16).cuda()
    tokens = torch.randint(0, V, (M, n), generator=g, dtype=torch.int32).cuda()
    mask = (torch.rand(M, generator=g) > 0.3).to(torch.uint8).cuda()
    return W, H, tokens, mask, torch.randn(M, n, generator=g).cuda() / M, torch.randn(M, k, generator=g).cuda() / M, \
        torch.randn(M, generator=g).cuda() / M


@pytest.mark.parametrize("M,K,V,n,k", [(1, 256, 1000, 1, 20), (7, 130, 1003, 2, 5), (53, 512, 5000, 1, 1), (600, 384, 2000, 1, 8)])
def test_scores_and_gradient_match_the_definitions(P, M, K, V, n, k):
    from paper_2403_17031_b200.pipeline import Fp8LMHead
    W, H, tokens, mask, g, gt, dh = _setup(M, K, V, n, k)
    head = Fp8LMHead(W, M, k, 0.7, n=n, backward=True)
    o = head.score(H, tokens, mask)
    wq, ws = F.quantize(W.float().cpu().numpy().T.copy(), 128)
    hq, hs = F.quantize(H.float().cpu().numpy(), 1)
    z, size = F.matmul(hq, hs, wq, ws, 128)
    logits = head.logits.double().cpu().numpy()
    gamma = (128 + -(-K // 128) + 3) * 2.0 ** -23
    assert (np.abs(logits - z) <= 2.0 ** -8 * np.abs(z) + gamma * size).all()
    want = T.topk(logits, npy(tokens), k, np.float32(0.7), npy(mask))
    assert np.array_equal(npy(o["top_ids"]), want["top_ids"])
    for name in ("logprob", "entropy", "lse", "top_logprob"):
        assert np.abs(npy(o[name]) - want[name]).max() <= TOL_LOGPROB, name
    lse, ent = npy(o["lse"]), npy(o["entropy"])
    dH = head.grad_hidden(tokens, g, gt, dentropy=dh, mask=mask)
    real = npy(mask).astype(bool)
    ids = np.where(real[:, None], np.concatenate([npy(tokens), want["top_ids"]], 1), 0)
    d, dsize = T.topk_bwd(logits, ids, np.concatenate([npy(g), npy(gt)], 1), lse, np.float32(0.7), ent, npy(dh), None, npy(mask))
    dl = head.dlogits.double().cpu().numpy()
    assert (np.abs(dl - d) <= 2.0 ** -8 * np.abs(d) + 4e-6 * dsize + 1e-38).all()
    dq, ds = F.quantize(head.dlogits.float().cpu().numpy(), 1)
    w2, w2s = F.quantize(W.float().cpu().numpy(), 128)
    y, ysize = F.matmul(dq, ds, w2, w2s, 128)
    gamma = (128 + -(-V // 128) + 3) * 2.0 ** -23
    assert (np.abs(dH.double().cpu().numpy() - y) <= 2.0 ** -8 * np.abs(y) + gamma * ysize + 1e-38).all()
    assert not npy(dH.float())[~real].any() and head.device_status() == 0


def test_capture_replay_and_two_heads_on_two_streams(P):
    from paper_2403_17031_b200.pipeline import Fp8LMHead
    M, K, V, k = 40, 512, 6000, 10
    W, H, tokens, mask, g, gt, dh = _setup(M, K, V, 1, k)
    heads = [Fp8LMHead(W if i == 0 else (W * 2).contiguous(), M, k, 1.0, backward=True) for i in range(2)]
    wants = []
    for h in heads:
        o = {n: v.clone() for n, v in h.score(H, tokens).items()}
        wants.append((o, h.grad_hidden(tokens, g, gt).clone()))
    assert not torch.equal(wants[0][1], wants[1][1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs = []
    for h, s in zip(heads, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            h.score(H, tokens)
            h.grad_hidden(tokens, g, gt)
        graphs.append(graph)
    for _ in range(3):
        for h in heads:
            h.dhidden.zero_()
            h.out["top_ids"].zero_()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):                  # both in flight at a time
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for h, (o, dH) in zip(heads, wants):
            assert all(torch.equal(h.out[n], o[n]) for n in o) and torch.equal(h.dhidden, dH)


def test_eight_bit_scores_are_near_the_bf16_heads(P):
    """Against the fused bf16 LM head on the same inputs: e4m3 is off by at most 2^-4 per factor, so a logit of K products of
    independent errors is off by about sqrt(K) * 0.04 * |h w| (rms of a relative error uniform in +-2^-4 is 0.036, two factors);
    a log-prob differs by the logit's error and the lse's, which is smaller. Eight such deviations is the bound."""
    from paper_2403_17031_b200.pipeline import Fp8LMHead
    M, K, V = 128, 1024, 4096
    W, H, tokens, mask, *_ = _setup(M, K, V, 1, 1)
    head = Fp8LMHead(W, M, 1, 1.0)
    o = head.score(H, tokens)
    ws = P.new_workspace(P.lmhead_workspace_bytes(M, K, V))
    lp, ent, lse = P.lmhead_logprob_entropy(H, W, tokens[:, 0].contiguous(), 1.0, ws)
    sd = K ** 0.5 * 0.036 * 2 ** 0.5 * 0.1                      # rms |h| = 1, rms |w| = 0.1
    assert (o["logprob"][:, 0] - lp).abs().max() <= 8 * 2 ** 0.5 * sd
    assert (o["lse"] - lse).abs().max() <= 8 * sd


def test_gradient_keeps_to_the_mask_of_its_scores(P):
    """grad_hidden() without a mask, with the one of score() and with another one; scores without a mask afterwards."""
    from paper_2403_17031_b200.pipeline import Fp8LMHead
    M, K, V, k = 53, 256, 3000, 6
    W, H, tokens, mask, g, gt, dh = _setup(M, K, V, 1, k)
    mask *= 2                                                   # (anything but 0 is a row)
    real = mask.bool()
    assert 0 < int(real.sum()) < M
    head = Fp8LMHead(W, M, k, 0.7, backward=True)
    free = {n: v.clone() for n, v in head.score(H, tokens).items()}
    full = head.grad_hidden(tokens, g, gt, dentropy=dh).clone()
    for top in (gt, None):
        o = head.score(H, tokens, mask)
        assert torch.equal(o["top_ids"][real], free["top_ids"][real]) and (o["top_ids"][~real] == -1).all()
        a = head.grad_hidden(tokens, g, top, dentropy=dh).clone()
        assert torch.equal(head.grad_hidden(tokens, g, top, dentropy=dh, mask=mask), a)
        assert not a[~real].any() and a[real].any(1).all() and head.device_status() == 0
        if top is gt:
            assert torch.equal(a[real], full[real])
        fewer = mask.clone().view(1, M)
        fewer[0, :M // 2] = 0
        fewer[0, M // 2:] = 1                                   # (the masked ones among these have no scores either)
        b = head.grad_hidden(tokens, g, top, dentropy=dh, mask=fewer)
        both = real & fewer[0].bool()
        assert torch.equal(b[both], a[both]) and not b[~both].any() and head.device_status() == 0
    for wrong, error in ((mask[:-1], ValueError), (mask.float(), TypeError), (mask.cpu(), TypeError)):
        with pytest.raises(error):
            head.grad_hidden(tokens, g, gt, mask=wrong)
        with pytest.raises(error):
            head.score(H, tokens, wrong)
    head.score(H, tokens)
    assert torch.equal(head.grad_hidden(tokens, g, gt, dentropy=dh), full)
    # a graph takes the mask as it is at its replay
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        head.score(H, tokens, mask)
        head.grad_hidden(tokens, g, gt, dentropy=dh)
    other = (torch.arange(M, device="cuda") % 3 != 0).to(torch.uint8)
    mask.copy_(other)
    head.score(H, tokens)                                       # (in between, without one)
    graph.replay()
    assert torch.equal(head.dhidden[other.bool()], full[other.bool()]) and not head.dhidden[~other.bool()].any()
    with pytest.raises(ValueError):
        Fp8LMHead(W, M, k, 0.7).grad_hidden(tokens, g)


def test_heads_whose_gradient_is_cut_along_the_vocabulary(P):
    """Scratch of more than its least size: the gradient's product against the product of whole tiles and the same call again; two heads
    in flight; captured."""
    from paper_2403_17031_b200.pipeline import Fp8LMHead
    M, K, V, k = 600, 2000, 12000, 4
    W, H, tokens, mask, g, gt, dh = _setup(M, K, V, 1, k)
    heads = [Fp8LMHead(W if i == 0 else (W * 0.5).contiguous(), M, k, 0.7, backward=True) for i in range(2)]
    assert P.fp8_scratch_bytes(M, K, V) > 256 and heads[0]._scratch_bwd.numel() == P.fp8_scratch_bytes(M, K, V)
    wants = []
    for h in heads:
        h.score(H, tokens, mask)
        wants.append(h.grad_hidden(tokens, g, gt, dentropy=dh).clone())
        y, size = F.matmul(npy(h.dlogits_q[0].float()), npy(h.dlogits_q[1]), npy(h.weight_bwd[0].float()), npy(h.weight_bwd[1]), 128)
        gamma = (128 + -(-V // 128) + 3) * 2.0 ** -23
        assert (np.abs(wants[-1].double().cpu().numpy() - y) <= 2.0 ** -8 * np.abs(y) + gamma * size + 1e-38).all()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs = []
    for h, s in zip(heads, streams):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            h.score(H, tokens, mask)
            h.grad_hidden(tokens, g, gt, dentropy=dh)
    for how in ("eager", "replayed", "replayed"):
        for h in heads:
            h.dhidden.zero_()
            h._scratch_bwd.fill_(255)
        torch.cuda.synchronize()
        for h, s, graph in zip(heads, streams, graphs):
            with torch.cuda.stream(s):
                if how == "eager":
                    h.score(H, tokens, mask)
                    h.grad_hidden(tokens, g, gt, dentropy=dh)
                else:
                    graph.replay()
        torch.cuda.synchronize()
        for h, w in zip(heads, wants):
            assert torch.equal(h.dhidden, w) and h.device_status() == 0, how


def test_eight_bit_gradient_is_near_the_bf16_heads(P):
    """dH_k = sum_v d_v W_kv against the bf16 head's, d the gradient of the token's log-prob. Off by, in standard deviations of independent
    errors: e4m3 (rms 0.036 relative) of d and W: 0.036 sqrt(2) sqrt(sum (d W)^2); d itself by p_v (e_v - sum p e) for logits off by e (rms
    `sd`, as for the scores above): at most 2 sd |g| sqrt(sum (p W)^2). Eight of either, and the roundings to bf16 on the way (the logits',
    half a step of |z| <= 16 moves p by 2^-5 and again by 2^-5 through lse: 2^-4 |g| sum p |W|; d's and the result's in either head: 2^-8
    of their terms each)."""
    from paper_2403_17031_b200.pipeline import Fp8LMHead
    M, K, V = 96, 512, 4096
    W, H, tokens, mask, g, *_ = _setup(M, K, V, 1, 1)
    head = Fp8LMHead(W, M, 0, 1.0, backward=True)
    head.score(H, tokens, mask)
    assert float(head.logits.abs().max()) <= 16
    got = head.grad_hidden(tokens, g).double()
    tok = tokens[:, 0].contiguous()
    ws = P.new_workspace(P.lmhead_workspace_bytes(M, K, V))
    _, _, lse = P.lmhead_logprob_entropy(H, W, tok, 1.0, ws)
    want = P.lmhead_bwd(H, W, tok, lse, g[:, 0].contiguous(), 1.0, ws, mask=mask, want_dW=False)["dH"].double()
    real = mask.bool()
    assert not got[~real].any() and not want[~real].any()
    w2 = W.double()
    p = torch.softmax(H.double() @ w2, 1)
    d = -p * g.double()
    d[torch.arange(M, device="cuda"), tok.long()] += g[:, 0].double()
    sd = K ** 0.5 * 0.036 * 2 ** 0.5 * 0.1
    absg = g.double().abs()
    bound = 8 * (0.036 * 2 ** 0.5 * (d * d @ (w2 * w2).t()).sqrt() + 2 * sd * absg * (p * p @ (w2 * w2).t()).sqrt())
    bound += 2.0 ** -4 * absg * (p @ w2.abs().t()) + 4 * 2.0 ** -8 * (d.abs() @ w2.abs().t())
    assert ((got - want).abs() <= bound)[real].all()
