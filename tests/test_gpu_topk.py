"""ppo_logprob_topk and its gradient against oracle/topk_oracle.py.

Ids are whole numbers decided by comparing stored logits: exact. Log-probs, entropy and lse: the library's tolerance for these
quantities. Gradients: half a step of the output type, relative, and 4e-6 of the sum of the absolute terms (fp32 evaluation: the
exponent is off by at most 2^-24 of |log2 p| <= 40 after its two-part subtraction, which is 1.7e-6 of p; ex2.approx 2^-22; the sum of
up to 256 gradients in a tree of 32 + 8 steps 2^-24 * 16 at the most)."""
import numpy as np
import pytest
import torch

from oracle import topk_oracle as O
from parity import TOL_LOGPROB, npy

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TAU = 0.7


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    import paper_2403_17031_b200 as pkg
    from paper_2403_17031_b200 import build
    build.build()
    pkg.lib()
    return pkg


def _logits(rows, V, dtype, pad=0, skip=0, seed=0, scale=3.0):
    """[rows, V] with a row pitch of V + pad elements, starting `skip` elements behind an aligned address."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.zeros(rows * (V + pad) + skip, dtype=dtype, device="cuda")
    x = flat[skip:].view(rows, V + pad)[:, :V]
    x.copy_((torch.randn(rows, V, generator=g) * scale).to(dtype))
    return x


def _same(got, want, what):
    """|d| <= TOL_LOGPROB + 2^-23 |want| where finite; NaN and infinities at the same places. The second term: an fp32 output of
    size w is rounded by up to 2^-24 w (1.2e-4 for an lse of 2857, so no fp32 result can meet the first term there), and the one
    rounded constant of the kernel, log2(e) / temperature, scales every exponent by another 2^-24."""
    got, want = npy(got).astype(np.float64), np.asarray(want)
    assert got.shape == want.shape, what
    fine = np.isfinite(want)
    with np.errstate(over="ignore"):
        far = fine & (np.abs(want) > 1e30)                       # (values that fp32 rounds to an infinity may be one)
        assert np.array_equal(np.isnan(got), np.isnan(want)), what
        assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
        near = fine & ~far
        d = np.abs(got[near] - want[near])
        assert (d <= TOL_LOGPROB + 2.0 ** -23 * np.abs(want[near])).all(), "%s: %.3e" % (what, d.max())
        rel = np.abs(got[far] / want[far] - 1)
        assert not rel.size or (rel <= 1e-6).all() or np.isinf(got[far]).all(), what


def _check(P, x, tokens, k, tau=TAU, mask=None, status=0):
    rows, V = x.shape
    ws = P.new_workspace(P.workspace_bytes(rows, 1, V))
    o = P.logprob_topk(x, tokens, k, tau, mask=mask, workspace=ws)
    torch.cuda.synchronize()
    assert P.last_device_status(ws) == status
    tok = npy(tokens).reshape(rows, -1)
    w = O.topk(x.double().cpu().numpy(), tok, k, np.float32(tau), None if mask is None else npy(mask))
    if k:
        assert np.array_equal(npy(o["top_ids"]), w["top_ids"]), "top_ids"
        _same(o["top_logprob"], w["top_logprob"], "top_logprob")
    _same(o["logprob"].reshape(rows, -1), w["logprob"], "logprob")
    _same(o["entropy"], w["entropy"], "entropy")
    _same(o["lse"], w["lse"], "lse")
    return o


def _tokens(rows, V, n=1, seed=1):
    return torch.randint(0, V, (rows, n), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype,rows,V,k,n,pad,skip", [
    (F32, 1, 1, 1, 1, 0, 0), (BF16, 3, 5, 5, 2, 0, 0), (BF16, 2, 17, 3, 1, 3, 5), (F32, 333, 70, 70, 1, 0, 1),
    (BF16, 300, 2048, 128, 1, 0, 0), (F32, 7, 1001, 128, 4, 3, 0), (BF16, 9, 1003, 17, 1, 1, 3), (BF16, 200, 1038, 128, 1, 0, 7),
    (BF16, 1, 50304, 20, 1, 0, 0), (BF16, 40, 50304, 1, 1, 0, 0), (F32, 60, 50277, 64, 128, 0, 0), (BF16, 2, 131080, 64, 1, 0, 0),
    (F32, 150, 4100, 33, 1, 0, 0), (BF16, 75, 32001, 8, 1, 0, 0), (BF16, 149, 50277, 5, 1, 0, 0), (F32, 37, 9000, 128, 1, 1, 1),
    (BF16, 36, 17000, 100, 1, 0, 2)])
def test_topk_matches_oracle(P, dtype, rows, V, k, n, pad, skip):
    _check(P, _logits(rows, V, dtype, pad, skip), _tokens(rows, V, n), k)


@pytest.mark.parametrize("rows", [1, 30, 60, 100, 300])
def test_topk_every_split_of_a_row_agrees_on_a_batch_of_equal_rows(P, rows):
    """The number of rows decides over how many blocks a row is split; ids must not depend on it."""
    x = _logits(1, 50304, BF16, seed=5).expand(rows, -1).contiguous()
    o = _check(P, x, _tokens(1, 50304).expand(rows, -1).contiguous(), 50)
    assert (o["top_ids"] == o["top_ids"][:1]).all() and (o["lse"] == o["lse"][:1]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows_each,V", [(1, 50304), (3, 20001), (30, 9001)])
def test_topk_rows_where_selection_is_hard(P, dtype, rows_each, V):
    base = _logits(12 * rows_each, V, dtype, seed=7)
    low = torch.finfo(dtype).min
    for i in range(rows_each):
        r = i * 12
        base[r] = 0.25                                        # every value equal: the lowest indices
        base[r + 1] = -torch.inf
        base[r + 1, V - 5:V - 2] = torch.tensor([1.0, 2.0, 1.0])   # fewer than k logits left
        base[r + 2] = low
        base[r + 2, 100:104] = 3.0                             # masked with the type's lowest value
        base[r + 3, 7] = -torch.inf
        base[r + 3, V // 2] = low
        base[r + 4] = torch.linspace(-20, 20, V, device="cuda").to(dtype)     # everything in one segment's reach, sorted
        base[r + 5] = torch.linspace(20, -20, V, device="cuda").to(dtype)
        base[r + 6] = (torch.arange(V, device="cuda") % 3).to(dtype)          # many ties at the threshold
        base[r + 7] = 0.0
        base[r + 7, ::2] = -0.0                                # equal values of either sign
        base[r + 8, 0] = 300.0                                 # one token holds everything
        base[r + 9] *= 20
        base[r + 9, V - 1] = 2000.0                            # far above the first pack: sums overflow at first
        base[r + 10, :8] = -torch.inf
        base[r + 11, 40:] = -torch.inf
    _check(P, base, _tokens(12 * rows_each, V, 2), 64)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(3, 50304), (40, 30001), (200, 9001), (700, 4100)])
def test_topk_rows_far_from_zero_with_banned_stretches(P, dtype, rows, V):
    """Logits around -400 (2^-800 of anything near 0) with the first, the last or every other thousand of them banned."""
    x = _logits(rows, V, dtype, seed=3, scale=2.0)
    x -= 400
    x[0::3, :min(3000, V - 40)] = -torch.inf
    x[1::3, -3000:-1] = torch.finfo(dtype).min
    x[2::3] = torch.where((torch.arange(V, device="cuda") // 1000) % 2 == 0, -torch.inf, x[2::3].float()).to(dtype)
    _check(P, x, _tokens(rows, V), 30)
    f = P.logprob_topk(x, None, 30, TAU)
    d = P.logprob_topk_bwd(x, f["lse"], TAU, top_ids=f["top_ids"], dtop_logprob=torch.ones(rows, 30, device="cuda"),
                           entropy=f["entropy"], dentropy=torch.ones(rows, device="cuda"))["dlogits"]
    assert torch.isfinite(d).all() and (d[0, :30] == 0).all()


def test_topk_takes_numbers_of_other_kinds(P):
    x = _logits(5, 600, F32)
    a, b = P.logprob_topk(x, None, np.int64(3), np.float32(0.7)), P.logprob_topk(x, None, 3, float(np.float32(0.7)))
    assert torch.equal(a["top_logprob"], b["top_logprob"])


def test_topk_rows_without_a_distribution(P):
    x = _logits(6, 5000, F32)
    x[0, 4321] = torch.nan
    x[1, 0] = torch.inf
    x[2] = -torch.inf
    x[3] = torch.finfo(F32).min
    x[5, 4999] = torch.nan
    _check(P, x, _tokens(6, 5000), 9, status=8)


def test_topk_mask_tokens_out_of_range_and_no_lists(P):
    x = _logits(50, 3001, BF16)
    mask = (torch.arange(50) % 3 != 0).to(torch.uint8).cuda()
    x[0] = torch.nan                                           # a masked row is not read
    _check(P, x, _tokens(50, 3001), 10, mask=mask)
    _check(P, x, _tokens(50, 3001), 10, mask=torch.zeros(50, dtype=torch.uint8, device="cuda"))
    tok = _tokens(50, 3001, 3)
    tok[4, 1], tok[5, 0] = 3001, -1
    _check(P, _logits(50, 3001, BF16), tok, 4, status=1)
    o = P.logprob_topk(_logits(50, 3001, BF16), None, 4, TAU)
    assert o["logprob"] is None and o["top_ids"].shape == (50, 4)
    o = P.logprob_topk(_logits(50, 3001, BF16), tok[:, 0].contiguous(), 0, TAU)
    assert o["top_ids"] is None and o["logprob"].shape == (50,)
    e = P.logprob_topk(_logits(50, 3001, BF16)[:0], None, 4, TAU)
    assert e["top_ids"].shape == (0, 4)


def test_topk_agrees_with_the_plain_call_and_repeats_bit_for_bit(P):
    x, tok = _logits(64, 50304, BF16), _tokens(64, 50304)[:, 0].contiguous()
    a, b = P.logprob_topk(x, tok, 20, TAU), P.logprob_topk(x, tok, 20, TAU)
    for name in a:
        assert torch.equal(a[name], b[name]), name
    lp, ent, lse = P.logprob_entropy(x, tok, TAU, want_lse=True)
    for got, want in ((a["logprob"], lp), (a["entropy"], ent), (a["lse"], lse)):
        assert (got - want).abs().max() <= 2 * TOL_LOGPROB


def test_topk_shapes_refusals_and_out(P):
    x = _logits(12, 900, F32).view(3, 4, 900)
    o = P.logprob_topk(x, _tokens(12, 900).view(3, 4), 6, TAU)
    assert o["logprob"].shape == (3, 4) and o["top_ids"].shape == (3, 4, 6) and o["lse"].shape == (3, 4)
    again = {n: torch.empty_like(v) for n, v in o.items()}
    assert P.logprob_topk(x, _tokens(12, 900).view(3, 4), 6, TAU, out=again) is again
    assert all(torch.equal(again[n], o[n]) for n in o)
    with pytest.raises(ValueError):
        P.logprob_topk(x, _tokens(11, 900), 6, TAU)
    with pytest.raises(ValueError):
        P.logprob_topk(x, _tokens(12, 900), 5, TAU, out=o)
    with pytest.raises(ValueError):
        P.logprob_topk(x, None, 6, TAU, mask=torch.ones(11, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        P.logprob_topk(x.transpose(0, 1), None, 6, TAU)
    with pytest.raises(TypeError):
        P.logprob_topk(x, _tokens(12, 900).long(), 6, TAU)
    with pytest.raises(P.PPOError):
        P.logprob_topk(x, None, 129, TAU)


def _bwd_inputs(rows, V, n, k, seed=3):
    g = torch.Generator().manual_seed(seed)
    top = torch.randint(0, V, (rows, k), generator=g, dtype=torch.int32)
    tok = torch.randint(0, V, (rows, n), generator=g, dtype=torch.int32)
    if n and k:
        top[:, 0] = tok[:, 0]                                  # given twice
    r = lambda *s: torch.randn(*s, generator=g).cuda()         # noqa: E731
    return tok.cuda(), r(rows, n), top.cuda(), r(rows, k), r(rows), r(rows)


def _check_bwd(P, x, n, k, tau=TAU, mask=None, entropy_grad=True, dlogits=None):
    rows, V = x.shape
    tok, g, top, gt, dh, dl = _bwd_inputs(rows, V, n, k)
    f = P.logprob_topk(x, None, 0, tau, mask=mask)
    more = dict(entropy=f["entropy"], dentropy=dh, dlse=dl) if entropy_grad else {}
    d = P.logprob_topk_bwd(x, f["lse"], tau, tokens=tok if n else None, dlogprob=g if n else None, top_ids=top if k else None,
                           dtop_logprob=gt if k else None, mask=mask, dlogits=dlogits, **more)["dlogits"]
    ids, gg = torch.cat([tok, top], 1), torch.cat([g, gt], 1)
    w, size = O.topk_bwd(x.double().cpu().numpy(), npy(ids), npy(gg), npy(f["lse"]), np.float32(tau),
                         npy(f["entropy"]) if entropy_grad else None, npy(dh) if entropy_grad else None,
                         npy(dl) if entropy_grad else None, None if mask is None else npy(mask))
    got = d.double().cpu().numpy()
    half = torch.finfo(x.dtype).eps / 2
    assert np.isfinite(got).all()
    assert (np.abs(got - w) <= half * np.abs(w) + 4e-6 * size + 1e-38).all(), np.abs(got - w).max()
    return d


@pytest.mark.parametrize("dtype,rows,V,n,k,pad,skip", [
    (F32, 1, 1, 1, 0, 0, 0), (BF16, 3, 5, 1, 5, 0, 0), (BF16, 4, 23, 2, 9, 1, 3), (F32, 9, 1001, 1, 128, 3, 0), (BF16, 5, 50277, 128, 128, 0, 0),
    (BF16, 53, 50304, 1, 20, 0, 0), (F32, 33, 4100, 4, 0, 0, 2), (BF16, 200, 8192, 1, 5, 8, 0), (F32, 3, 131072, 0, 64, 0, 0),
    (BF16, 2, 8199, 0, 0, 0, 1)])
def test_topk_bwd_matches_oracle(P, dtype, rows, V, n, k, pad, skip):
    x = _logits(rows, V, dtype, pad, skip)
    if V > 2:
        x[:, V - 2] = -torch.inf
    _check_bwd(P, x, n, k)
    _check_bwd(P, x, n, k, entropy_grad=False)


def test_topk_bwd_masked_rows_strided_output_and_bits(P):
    rows, V = 40, 5003
    x = _logits(rows, V, BF16, pad=5)
    mask = (torch.arange(rows) % 4 != 1).to(torch.uint8).cuda()
    x[1] = torch.nan                                           # a masked row is not read
    buf = torch.full((rows, V + 9), 7.0, dtype=BF16, device="cuda")
    a = _check_bwd(P, x, 1, 6, mask=mask, dlogits=buf[:, :V]).clone()
    assert (buf[:, V:] == 7.0).all() and (a[1] == 0).all()     # what lies behind a row stays as it was
    assert torch.equal(a, _check_bwd(P, x, 1, 6, mask=mask))


def test_topk_bwd_bad_ids_and_nan_rows(P):
    rows, V = 8, 9000
    x = _logits(rows, V, F32)
    tok, g, top, gt, dh, dl = _bwd_inputs(rows, V, 1, 4)
    f = P.logprob_topk(x, None, 0, TAU)
    top[3, 2] = V
    f["lse"][5] = torch.nan
    ws = P.new_workspace(P.workspace_bytes(rows, 1, V))
    d = P.logprob_topk_bwd(x, f["lse"], TAU, tokens=tok, dlogprob=g, top_ids=top, dtop_logprob=gt, workspace=ws)["dlogits"]
    assert P.last_device_status(ws) == 1
    nan = torch.isnan(d)
    assert nan[3].all() and nan[5].all() and not nan[[0, 1, 2, 4, 6, 7]].any()


def test_topk_bwd_gradient_matches_differences_of_the_forward_call(P):
    """Central differences of the library's own forward results along random directions (fp32, fp64 sums on the host)."""
    rows, V, k = 3, 600, 5
    x = _logits(rows, V, F32, scale=1.0)
    tok, g, _, gt, dh, dl = _bwd_inputs(rows, V, 1, k)
    f = P.logprob_topk(x, tok, k, 1.0)
    ids = torch.cat([tok, f["top_ids"]], 1).contiguous()
    gg = torch.cat([g, gt], 1).contiguous()

    def value(y):
        o = P.logprob_topk(y, ids, 0, 1.0)
        return float((o["logprob"].double() * gg).sum() + (o["entropy"].double() * dh).sum() + (o["lse"].double() * dl).sum())
    d = P.logprob_topk_bwd(x, f["lse"], 1.0, tokens=tok, dlogprob=g, top_ids=f["top_ids"], dtop_logprob=gt, entropy=f["entropy"],
                           dentropy=dh, dlse=dl)["dlogits"].double()
    for seed in range(4):
        u = torch.randn(rows, V, generator=torch.Generator().manual_seed(seed)).cuda()
        h = 2.0 ** -6
        diff = (value(x + h * u) - value(x - h * u)) / (2 * h)
        # each of ~25 outputs is off by at most 1e-5 relative to a gradient of order 1 (fp32 sums of 600 terms): 25e-5 / (2 h) = 0.008;
        # curvature: h^2 / 6 times third derivatives of order |u|^3 p <= 0.01
        assert abs(diff - float((d * u).sum())) <= 0.02 + 0.01 * abs(diff)


def test_topk_on_another_stream_and_in_a_graph(P):
    x, tok = _logits(20, 50304, BF16), _tokens(20, 50304)
    want = P.logprob_topk(x, tok, 20, TAU)
    out = {n: torch.zeros_like(v) for n, v in want.items()}
    d = torch.zeros_like(x)
    g, gt = torch.ones(20, 1, device="cuda"), torch.ones(20, 20, device="cuda")

    def both():
        P.logprob_topk(x, tok, 20, TAU, out=out)
        P.logprob_topk_bwd(x, out["lse"], TAU, tokens=tok, dlogprob=g, top_ids=out["top_ids"], dtop_logprob=gt, dlogits=d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    s.synchronize()
    assert all(torch.equal(out[n], want[n]) for n in want)
    first = d.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for t in (*out.values(), d):
        t.zero_()
    x2 = _logits(20, 50304, BF16, seed=9)
    keep = x.clone()
    x.copy_(x2)
    graph.replay()
    assert torch.equal(out["top_ids"], P.logprob_topk(x2, tok, 20, TAU)["top_ids"]) and not torch.equal(d, first)
    x.copy_(keep)
    graph.replay()
    assert all(torch.equal(out[n], want[n]) for n in want) and torch.equal(d, first)


def test_topk_offsets_past_32_bits(P):
    """A batch whose elements lie beyond 2^32: the last rows are right (bf16, 4.4e9 elements)."""
    V, rows = 50304, 88000
    x = torch.zeros(rows, V, dtype=BF16, device="cuda")
    tail = _logits(4, V, BF16, seed=11)
    x[-4:] = tail
    mask = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    mask[-4:] = 1
    tok = _tokens(rows, V)
    o = P.logprob_topk(x, tok, 7, TAU, mask=mask)
    w = P.logprob_topk(tail, tok[-4:].contiguous(), 7, TAU)
    assert torch.equal(o["top_ids"][-4:], w["top_ids"]) and (o["top_ids"][:-4] == -1).all()
    assert (o["lse"][-4:] - w["lse"]).abs().max() <= TOL_LOGPROB
    d = P.logprob_topk_bwd(x, o["lse"], TAU, tokens=tok, dlogprob=torch.ones(rows, 1, device="cuda"), mask=mask)["dlogits"]
    dt = P.logprob_topk_bwd(tail, o["lse"][-4:].contiguous(), TAU, tokens=tok[-4:].contiguous(), dlogprob=torch.ones(4, 1, device="cuda"))
    assert torch.equal(d[-4:], dt["dlogits"]) and not d[:1000].any()


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("rows,V", [(600, 32768), (600, 30011), (2, 50304)])
def test_best_elements_at_regular_distances(P, dt, rows, V):
    """The k best, all different, at one distance from each other: few or many of them in the same thread's share."""
    g = torch.Generator(device="cuda").manual_seed(11)
    x = torch.rand(rows, V, device="cuda", generator=g).mul(4).to(dt)            # all below 8
    n = 8 if dt == BF16 else 4
    dists = [1, n, 16 * n, 32 * n, 256 * n, 257 * n, 512 * n, 128 * n + 1]
    k = 7
    ids = torch.empty(rows, k, dtype=torch.int64)
    for r in range(rows):
        d = dists[r % len(dists)]
        ids[r] = (torch.arange(k) * d + 37 * r) % V
    assert all(len(set(row.tolist())) == k for row in ids)
    ids = ids.cuda()
    x.scatter_(1, ids, torch.arange(8 + k, 8, -1, device="cuda").to(dt).expand(rows, k))     # exact in both types
    o = P.logprob_topk(x, None, k, 1.0)
    assert torch.equal(o["top_ids"].long(), ids)
    full = P.logprob_topk(x, None, 100, 1.0)["top_ids"].long()
    want = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :100]
    assert torch.equal(full, want)


@pytest.mark.parametrize("dtype,rows,V,k,n,pad,skip", [
    (F32, 600, 1, 1, 1, 0, 0), (BF16, 700, 7, 7, 2, 1, 1), (BF16, 601, 33, 32, 1, 0, 3), (F32, 600, 513, 32, 128, 3, 1),
    (BF16, 1500, 1025, 31, 1, 0, 0), (F32, 600, 8190, 20, 1, 0, 0), (BF16, 600, 16391, 5, 1, 1, 0), (BF16, 600, 16400, 5, 1, 0, 0),
    (F32, 592, 4100, 33, 1, 0, 0), (BF16, 591, 4100, 32, 1, 0, 0), (BF16, 600, 4100, 0, 1, 0, 0)])
def test_topk_of_many_rows_of_little_length(P, dtype, rows, V, k, n, pad, skip):
    """(either side of 592 rows, 16384 bf16 elements and 32 alternatives, where blocks of another size take over)"""
    mask = (torch.arange(rows) % 3 != 1).to(torch.uint8).cuda()
    _check(P, _logits(rows, V, dtype, pad, skip, seed=9), _tokens(rows, V, n), k, mask=mask)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [150, 1200, 8001])
def test_many_short_rows_where_selection_is_hard(P, dtype, V):
    base = _logits(600, V, dtype, seed=8)
    low = torch.finfo(dtype).min
    at = torch.arange(V, device="cuda")
    base[0::12] = 0.25
    base[1::12] = -torch.inf
    base[1::12, V - 5:V - 2] = torch.tensor([1.0, 2.0, 1.0], device="cuda", dtype=dtype)
    base[2::12] = low
    base[2::12, 100:104] = 3.0
    base[3::12, 7] = -torch.inf
    base[3::12, V // 2] = low
    base[4::12] = torch.linspace(-20, 20, V, device="cuda").to(dtype)
    base[5::12] = torch.linspace(20, -20, V, device="cuda").to(dtype)
    base[6::12] = (at % 3).to(dtype)
    base[7::12] = 0.0
    base[7::12, ::2] = -0.0
    base[8::12, 0] = 300.0
    base[9::12] *= 20
    base[9::12, V - 1] = 2000.0
    base[10::12, :8] = -torch.inf
    base[11::12, 40:] = -torch.inf
    _check(P, base, _tokens(600, V, 2), 32)


def test_many_short_rows_without_a_distribution(P):
    x = _logits(600, 2000, BF16, seed=10)
    x[5, 3] = torch.nan
    x[6, 1999] = torch.inf
    x[7] = -torch.inf
    ws = P.new_workspace(P.workspace_bytes(600, 1, 2000))
    o = P.logprob_topk(x, _tokens(600, 2000)[:, 0].contiguous(), 9, TAU, workspace=ws)
    torch.cuda.synchronize()
    assert P.last_device_status(ws) == 8
    bad = torch.zeros(600, dtype=torch.bool, device="cuda")
    bad[5:8] = True
    assert (o["top_ids"][bad] == -1).all() and (o["top_ids"][~bad] >= 0).all()
    for name in ("logprob", "entropy", "lse"):
        assert torch.equal(torch.isnan(o[name]), bad), name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(9, 50304), (60, 20011), (130, 9001), (9, 131080)])
@pytest.mark.parametrize("k", [32, 100, 128])
def test_few_rows_with_many_alternatives_and_banned_stretches(P, dtype, rows, V, k):
    """The blocks that share a row agree on a threshold; some of them, or all, may have fewer than their part of the k."""
    x = _logits(rows, V, dtype, seed=12)
    at = torch.arange(V, device="cuda")
    x[0::9, :V // 8 + 20] = -torch.inf                      # the first of eight blocks
    x[1::9, V // 4:] = -torch.inf                           # all but two of eight
    x[2::9, 60:] = -torch.inf                               # fewer than k left in all, all of them in the first block
    x[3::9] = torch.where(at % (V // 70) == 0, x[3::9].float(), -torch.inf).to(dtype)     # about 70 left, everywhere
    x[4::9, V // 2:] = torch.finfo(dtype).min
    x[5::9, V // 8:V // 8 + 20] += 30                       # the best of them in one block
    x[6::9] = torch.where((at < V // 2) | (at > V - 40), x[6::9].float(), -torch.inf).to(dtype)   # a few in the last block
    x[7::9] = -torch.inf
    x[7::9, V - 1] = 1.0
    _check(P, x, _tokens(rows, V), k)


def test_nan_in_one_block_of_a_shared_row(P):
    x = _logits(2, 50304, BF16, seed=13)
    x[0, 40000] = torch.nan
    for k in (5, 64):
        o = P.logprob_topk(x, None, k, TAU)
        assert (o["top_ids"][0] == -1).all() and torch.isnan(o["lse"][0])
        want = torch.sort(x[1].float(), descending=True, stable=True).indices[:k]
        assert torch.equal(o["top_ids"][1].long(), want)


@pytest.mark.parametrize("rows", [36, 73, 148, 149, 250, 296, 297])
def test_topk_of_long_fp32_rows_at_every_split(P, rows):
    x = _logits(rows, 32801, F32, seed=14)
    _check(P, x, _tokens(rows, 32801), 33)


def _hard_rows(V, dtype, seed):
    """Twelve kinds of rows: equal, tied, sorted, peaked or mostly banned values."""
    base = _logits(12, V, dtype, seed=seed)
    at, low = torch.arange(V, device="cuda"), torch.finfo(dtype).min
    base[0] = 0.25
    base[1] = -torch.inf
    base[1, V - 5:V - 2] = torch.tensor([1.0, 2.0, 1.0], device="cuda", dtype=dtype)
    base[2] = low
    base[2, 100:104] = 3.0
    base[3, 7], base[3, V // 2] = -torch.inf, low
    base[4] = torch.linspace(-20, 20, V, device="cuda").to(dtype)
    base[5] = torch.linspace(20, -20, V, device="cuda").to(dtype)
    base[6] = (at % 3).to(dtype)
    base[7, ::2] = low
    base[8, 0] = 300.0
    base[9, V - 1] = 2000.0
    base[10, :V // 2] = -torch.inf
    base[11, 40:] = -torch.inf
    return base


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau", [1.5, 1.7, 2.0, 4.0, 8.0])
@pytest.mark.parametrize("each,V,pad,skip", [(1, 50304, 0, 0), (3, 20001, 0, 1), (10, 9001, 0, 0), (20, 9001, 3, 2), (60, 4100, 0, 0)])
def test_banned_stretches_at_high_temperatures(P, dtype, tau, each, V, pad, skip):
    """Above log2(e) a masked logit times log2(e) / temperature lies nearer to 0 than the value it was clamped to. Each of the kernel's
    splits of a row (1, 2, 4 and 8 blocks, blocks of 128 threads), aligned and odd rows."""
    x = _logits(12 * each, V, dtype, pad, skip)
    x.copy_(_hard_rows(V, dtype, 15).repeat(each, 1))
    _check(P, x, _tokens(12 * each, V, 2), 30, tau=tau)
    x -= 400                                                   # (keeps -inf; bf16's lowest value stays where it is too)
    _check(P, x, _tokens(12 * each, V, 2), 30, tau=tau)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau", [1.5, 2.0, 2.8853900817779268])
def test_rows_without_a_distribution_at_high_temperatures(P, dtype, tau):
    """(the last temperature is 2 log2(e): its factor 0.5 scales exactly, without a rounding error that gives the row away)"""
    x = _logits(6, 5001, dtype)
    x[0, 4321] = torch.nan
    x[1, 0] = torch.inf
    x[2] = -torch.inf
    x[3] = torch.finfo(dtype).min
    x[5] = -torch.inf
    x[5, 5000] = torch.nan                                     # a NaN among nothing but banned logits
    _check(P, x, _tokens(6, 5001), 9, tau=tau, status=8)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau", [2.0, 8.0])
@pytest.mark.parametrize("rows,k", [(9, 20), (9, 128), (60, 64)])
def test_few_rows_with_banned_blocks_at_high_temperatures(P, dtype, tau, rows, k):
    V = 50304
    x = _logits(rows, V, dtype, seed=16)
    x[0::4, :V // 8 + 20] = -torch.inf
    x[1::4, V // 4:] = torch.finfo(dtype).min
    x[2::4, 60:] = -torch.inf
    x[3::4] = torch.where(torch.arange(V, device="cuda") % (V // 70) == 0, x[3::4].float(), -torch.inf).to(dtype)
    _check(P, x, _tokens(rows, V), k, tau=tau)


def _soft_masked_rows(V, dtype, base, best, seed):
    """[8, V]: all logits at `base` but for some hundreds at 0, in the whole row or its second half, and one at `best`."""
    g = torch.Generator().manual_seed(seed)
    x = torch.full((8, V), float(base))
    for r in range(8):
        first = V // 2 if r >= 3 else 0
        x[r, first + torch.randperm(V - first, generator=g)[:V // 30]] = 0.0
        x[r, [0, V - 2, V // 2, 3][r % 4]] = best
    return x.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("each,V", [(1, 50304), (12, 9000), (40, 9001), (90, 4096)])
def test_logits_that_are_masked_softly(P, dtype, each, V):
    """Bases around 2^-126 of the rest: references of different warps so far apart that fp32 cannot scale one's sums to the other's."""
    for base, best in ((-60, 4.25), (-76, 12), (-78, 10), (-79, 9), (-80, 8), (-80, 12), (-82, 4.25), (-83.5, 4.25), (-85, 4.25), (-88, 4.25),
                       (-120, 4.25), (-300, 4.25)):
        x = _soft_masked_rows(V, dtype, base, best, 19).repeat(each, 1)
        _check(P, x, _tokens(8 * each, V), 20, tau=1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(24, 50304), (300, 9001)])
def test_logits_of_great_magnitude(P, dtype, rows, V):
    """Up to 7e8 temperature: as accurate as fp32 outputs of that size are; above: no distribution, in either direction. (The factor
    log2(e) / temperature is rounded to 24 bits, which moves a log-prob by up to 2^-24 of its logit: the second term of _same; here the
    terms of a log-prob are far larger than itself, so it is taken of those.)"""
    x = _logits(rows, V, dtype, seed=17, scale=1.0)
    scale = torch.tensor([1e3, 1e5, 1e7, 6e8, 1e9, 1e10, 1e13, 1e20], device="cuda").repeat(rows // 4)[:rows, None]
    sign = torch.where(torch.arange(rows, device="cuda") % 16 < 8, 1.0, -1.0)[:, None]
    x.copy_((x.float().abs() * 1e-4 + 0.9).clamp_max(1.0) * scale * sign)      # all of a row near its largest
    o = P.logprob_topk(x, _tokens(rows, V), 20, 1.0)
    bad = (x.float().max(1).values.abs() > 7.45e8).tolist()
    ids = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :20]
    z = x.double()
    w = z.logsumexp(1)
    assert any(bad) and not all(bad)
    for r in range(rows):
        if bad[r]:
            assert (o["top_ids"][r] == -1).all() and torch.isnan(o["lse"][r]) and torch.isnan(o["top_logprob"][r]).all(), r
            continue
        assert torch.equal(o["top_ids"][r].long(), ids[r]), r
        tol = TOL_LOGPROB + 2.0 ** -23 * float(w[r].abs())
        assert abs(float(o["lse"][r]) - float(w[r])) <= tol, r
        spread = float(z[r].max() - z[r].min())
        d = (o["top_logprob"][r].double() - (z[r][ids[r]] - w[r])).abs().max()
        assert float(d) <= TOL_LOGPROB + 2.0 ** -23 * spread, r


def test_rows_of_great_magnitude_at_a_tiny_temperature(P):
    """The same limit on logits / temperature, and masked logits whose quotient leaves fp32's range."""
    x = _logits(8, 9001, F32, seed=18, scale=1e-3)
    x[:, ::3] = -torch.inf
    x[::2, 1::3] = torch.finfo(F32).min
    for tau in (1e-6, 1e-9, 1e-11):
        _check(P, x, _tokens(8, 9001), 10, tau=tau)
    o = P.logprob_topk(x, None, 10, 1e-13)
    assert (o["top_ids"] == -1).all() and torch.isnan(o["lse"]).all()
