"""What the scoring and 8-bit LM-head operators of this library are measured on: the cases, their inputs, the
operators in plain torch operations, the library's own calls, and the same results in 64 bits.

  topk       ppo_logprob_topk      log-probs of given tokens, entropy, log-sum-exp and the k most likely alternatives
  topk_bwd   ppo_logprob_topk_bwd  gradients on all of those back to the logits
  quantize   ppo_fp8_quantize      bf16 / fp32 matrix to e4m3 with one scale per 1 x 128 or 128 x 128 block
  matmul     ppo_fp8_matmul        product of two such matrices, A [M,K] B[N,K]^T, scales applied block by block
"""
import math

import torch

own = False

TEMPERATURE = 0.7      # the paper's sampling temperature
E4M3_MAX = 448.0
MIN_AMAX = 2.0 ** -100   # a block whose largest magnitude is below this is scaled as if it were this


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of one sequence being decoded, with the alternatives a client shows beside it
        {"name": "topk 1x50304 bf16 k20", "op": "topk", "rows": 1, "V": 50304, "dtype": "bf16", "k": 20, "n": 1,
         "pad": 0, "T": 0},
        # a rollout batch of 64 responses x 53 tokens, padding after each response's first EOS masked out
        {"name": "topk 3392x50304 bf16 k5", "op": "topk", "rows": 3392, "V": 50304, "dtype": "bf16", "k": 5, "n": 1,
         "pad": 0, "T": 53},
        # teacher scores for distillation: fp32 logits of the unpadded vocabulary (rows at odd addresses), many
        # alternatives, and the log-probs of several given tokens
        {"name": "topk 997x50277 fp32 k64", "op": "topk", "rows": 997, "V": 50277, "dtype": "fp32", "k": 64, "n": 4,
         "pad": 0, "T": 0},
        # gradient of one response's token and top-20 log-probs with an entropy bonus
        {"name": "topk_bwd 53x50304 bf16 n21", "op": "topk_bwd", "rows": 53, "V": 50304, "dtype": "bf16", "k": 20,
         "n": 1, "pad": 0, "T": 0},
        # the same batch as above, masked, top 5
        {"name": "topk_bwd 3392x50304 bf16 n6", "op": "topk_bwd", "rows": 3392, "V": 50304, "dtype": "bf16", "k": 5,
         "n": 1, "pad": 0, "T": 53},
        # fp32 student logits of the unpadded vocabulary, 64 teacher alternatives and one token
        {"name": "topk_bwd 997x50277 fp32 n65", "op": "topk_bwd", "rows": 997, "V": 50277, "dtype": "fp32", "k": 64,
         "n": 1, "pad": 0, "T": 0},
        # hidden states of a rollout batch, one scale per row and 128 columns
        {"name": "quantize 3392x4096 rows", "op": "quantize", "M": 3392, "K": 4096, "dtype": "bf16", "block": 1,
         "transpose": False},
        # the LM head's weight [K, V] once per update, stored [V, K] with one scale per 128 x 128
        {"name": "quantize 4096x50304 block T", "op": "quantize", "M": 50304, "K": 4096, "dtype": "bf16",
         "block": 128, "transpose": True},
        # the LM head for one token being decoded
        {"name": "matmul 1x50304x4096", "op": "matmul", "M": 1, "N": 50304, "K": 4096, "block": 128, "out": "bf16"},
        # odd sizes in all three directions, fp32 result
        {"name": "matmul 300x1000x577 fp32", "op": "matmul", "M": 300, "N": 1000, "K": 577, "block": 128,
         "out": "fp32"},
        # gradient on the hidden states of a rollout batch: contraction over the vocabulary
        {"name": "matmul 3392x4096x50304", "op": "matmul", "M": 3392, "N": 4096, "K": 50304, "block": 128,
         "out": "bf16"},
        # logits of a full batch of 512 responses x 53 tokens
        {"name": "matmul 27136x50304x4096", "op": "matmul", "M": 27136, "N": 50304, "K": 4096, "block": 128,
         "out": "bf16"},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["topk", "topk_bwd", "quantize", "matmul"])
    if op in ("topk", "topk_bwd"):
        dtype = rng.choice(["bf16", "fp32"])
        T = rng.choice([0, 53])
        rows = _spread(rng, 1, 3392 if dtype == "bf16" else 1600)
        if T:
            rows = max(1, rows // T) * T
        V = rng.choice([50304, 50277, _spread(rng, 1000, 60000)])
        return {"op": op, "rows": rows, "V": V, "dtype": dtype, "k": _spread(rng, 1, 128), "n": rng.choice([1, 1, 4]),
                "pad": rng.choice([0, 0, 3, 8]), "T": T}
    if op == "quantize":
        return {"op": op, "M": _spread(rng, 1, 27136), "K": _spread(rng, 100, 6000), "dtype": rng.choice(["bf16", "fp32"]),
                "block": rng.choice([1, 128]), "transpose": rng.random() < 0.5}
    return {"op": op, "M": _spread(rng, 1, 6784), "N": _spread(rng, 100, 50304), "K": _spread(rng, 100, 8192),
            "block": rng.choice([1, 128, 128]), "out": rng.choice(["bf16", "fp32"])}


def work(case):
    op = case["op"]
    if op in ("topk", "topk_bwd"):
        size = 2 if case["dtype"] == "bf16" else 4
        real = case["rows"] * 0.5 * (1 + 1 / case["T"]) if case["T"] else case["rows"]    # lengths are uniform in 1..T
        ids = case["n"] + case["k"]
        if op == "topk":
            return {"bytes": real * case["V"] * size + case["rows"] * (8 * ids + 8), "flops": real * case["V"] * 6}
        return {"bytes": (real + case["rows"]) * case["V"] * size + case["rows"] * (8 * ids + 16),
                "flops": real * case["V"] * 6}
    if op == "quantize":
        size = 2 if case["dtype"] == "bf16" else 4
        blocks = -(-case["K"] // 128) * -(-case["M"] // case["block"])
        return {"bytes": case["M"] * case["K"] * (size + 1) + 4 * blocks, "flops": 3 * case["M"] * case["K"]}
    M, N, K = case["M"], case["N"], case["K"]
    kb = -(-K // 128)
    return {"bytes": M * K + N * K + 4 * kb * (M + -(-N // case["block"])) + M * N * (2 if case["out"] == "bf16" else 4),
            "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _quantized(x, block):
    """x [R, C] as the operator's 8-bit operand: values [R, C] at a row pitch that is a multiple of 16, and scales
    [ceil(C/128), R] (block 1) or [ceil(R/128), ceil(C/128)] (block 128)."""
    R, C = x.shape
    q, s = _plain_quantize(x, block)
    buf = torch.zeros((R, -(-C // 16) * 16), dtype=torch.float8_e4m3fn, device=x.device)
    buf[:, :C] = q
    return buf[:, :C], s


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *s: torch.rand(*s, generator=g, device=dev)        # noqa: E731
    randn = lambda *s: torch.randn(*s, generator=g, device=dev)      # noqa: E731
    op = case["op"]
    st = {"case": dict(case)}
    if op in ("topk", "topk_bwd"):
        rows, V, k, n = case["rows"], case["V"], case["k"], case["n"]
        x = randn(rows, V + case["pad"])
        x *= 0.5 + 3.5 * rand(rows, 1)                                # sharper and flatter rows
        x[:, 1] = -math.inf                                           # [PAD] is banned
        x = x.to(_dtype(case["dtype"]))[:, :V]
        st["logits"] = x
        st["mask"] = None
        if case["T"]:
            length = torch.randint(1, case["T"] + 1, (rows // case["T"], 1), generator=g, device=dev)
            st["mask"] = (torch.arange(case["T"], device=dev)[None] < length).to(torch.uint8).reshape(rows)
        tok = torch.randint(2, V, (rows, n), generator=g, device=dev)
        if op == "topk":
            st["tokens"] = tok.to(torch.int32)
            return st
        # the sampled token is one of the likely ones, so it is often among the alternatives
        lse, ent, top = [], [], []
        for part in x.split(256):                                     # what the forward call left behind
            z = part.double() / TEMPERATURE
            lp = z.log_softmax(1)
            lse.append(z.logsumexp(1).float())
            ent.append(-(lp.exp() * lp.masked_fill(lp == -math.inf, 0)).sum(1).float())
            top.append(z.topk(k, 1).indices)
        top = torch.cat(top)
        tok[:, 0] = top[:, 0]
        st["tokens"], st["top_ids"] = tok.to(torch.int32), top.to(torch.int32)
        st["lse"], st["entropy"] = torch.cat(lse), torch.cat(ent)
        st["dlogprob"], st["dtop"] = randn(rows, n) / rows, 0.2 * randn(rows, k) / rows
        st["dentropy"], st["dlse"] = -0.05 * rand(rows) / rows, 0.01 * randn(rows) / rows
        return st
    if op == "quantize":
        shape = (case["K"], case["M"]) if case["transpose"] else (case["M"], case["K"])
        x = randn(*shape)
        x *= 0.02 * (1 + 9 * rand(shape[0], 1))                       # rows of different magnitude
        st["x"] = x.to(_dtype(case["dtype"]))
        return st
    a, b = randn(case["M"], case["K"]), randn(case["N"], case["K"])
    b *= 0.02
    a *= 1 + 4 * rand(case["M"], 1)
    st["a"], st["a_scales"] = _quantized(a, 1)
    st["b"], st["b_scales"] = _quantized(b, case["block"])
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    op = st["case"]["op"]
    if own:
        return _OWN[op](st)
    return _PLAIN[op](st)


def _own_topk(st):
    from paper_2403_17031_b200 import binding as b
    return b.logprob_topk(st["logits"], st["tokens"], st["case"]["k"], TEMPERATURE, mask=st["mask"])


def _own_topk_bwd(st):
    from paper_2403_17031_b200 import binding as b
    return b.logprob_topk_bwd(st["logits"], st["lse"], TEMPERATURE, tokens=st["tokens"], dlogprob=st["dlogprob"],
                              top_ids=st["top_ids"], dtop_logprob=st["dtop"], entropy=st["entropy"],
                              dentropy=st["dentropy"], dlse=st["dlse"], mask=st["mask"])


def _own_quantize(st):
    from paper_2403_17031_b200 import binding as b
    q, s = b.fp8_quantize(st["x"], block_rows=st["case"]["block"], transpose=st["case"]["transpose"])
    return {"q": q, "scales": s}


def _own_matmul(st):
    from paper_2403_17031_b200 import binding as b
    return b.fp8_matmul(st["a"], st["a_scales"], st["b"], st["b_scales"], block_n=st["case"]["block"],
                        out_dtype=_dtype(st["case"]["out"]))


# ---- the plain forms
def _ordered_keys(x):
    """Whole numbers that order like (value descending, index ascending): larger is earlier."""
    bits = (x.float() + 0.0).view(torch.int32).long()                 # (-0 becomes +0)
    value = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    index = torch.arange(x.shape[1], device=x.device)
    return (value << 32) + (0xFFFFFFFF - index)


def _plain_topk(st):
    x, k, mask = st["logits"], st["case"]["k"], st["mask"]
    z = x.float() / TEMPERATURE
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    s = e.sum(1, keepdim=True)
    lse = top + torch.log(s)
    lp = z - lse
    entropy = -(e / s * torch.where(e > 0, lp, 0.0)).sum(1)
    ids = 0xFFFFFFFF - (_ordered_keys(x).topk(k, 1).values & 0xFFFFFFFF)
    out = {"logprob": lp.gather(1, st["tokens"].long()), "entropy": entropy, "lse": lse[:, 0],
           "top_ids": ids.to(torch.int32), "top_logprob": lp.gather(1, ids)}
    if mask is not None:                                              # masked rows: 0, and -1 for the ids
        off = mask == 0
        for name, v in out.items():
            v[off] = -1 if name == "top_ids" else 0
    return out


def _plain_topk_bwd(st):
    x, mask = st["logits"], st["mask"]
    lp = x.float() / TEMPERATURE - st["lse"][:, None]
    ids = torch.cat([st["tokens"], st["top_ids"]], 1).long()
    g = torch.cat([st["dlogprob"], st["dtop"]], 1)
    p = torch.exp(lp)
    slope = (st["dlse"] - g.sum(1))[:, None] - st["dentropy"][:, None] * (torch.where(p > 0, lp, 0.0) + st["entropy"][:, None])
    d = p * slope
    d.scatter_add_(1, ids, g)
    d /= TEMPERATURE
    if mask is not None:
        d[mask == 0] = 0
    return {"dlogits": d.to(x.dtype)}


def _plain_quantize(x, block):
    R, C = x.shape
    rb, cb = -(-R // block), -(-C // 128)
    full = torch.zeros((rb * block, cb * 128), dtype=torch.float32, device=x.device)
    full[:R, :C] = x
    full = full.view(rb, block, cb, 128)
    amax = full.abs().amax((1, 3)).clamp_min(MIN_AMAX)
    scales = amax / E4M3_MAX
    q = (full * (E4M3_MAX / amax)[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    q = q.view(rb * block, cb * 128)[:R, :C]
    return q, (scales.t().contiguous() if block == 1 else scales)


def _plain_quantize_case(st):
    x = st["x"].t() if st["case"]["transpose"] else st["x"]
    q, s = _plain_quantize(x, st["case"]["block"])
    return {"q": q, "scales": s}


def _plain_matmul(st):
    M, K = st["a"].shape
    N, block = st["b"].shape[0], st["case"]["block"]
    sa = st["a_scales"].t().repeat_interleave(128, 1)[:, :K]
    sb = st["b_scales"].t() if block == 1 else st["b_scales"].repeat_interleave(128, 0)[:N]
    sb = sb.repeat_interleave(128, 1)[:, :K]
    return ((st["a"].float() * sa) @ (st["b"].float() * sb).t()).to(_dtype(st["case"]["out"]))


_OWN = {"topk": _own_topk, "topk_bwd": _own_topk_bwd, "quantize": _own_quantize, "matmul": _own_matmul}
_PLAIN = {"topk": _plain_topk, "topk_bwd": _plain_topk_bwd, "quantize": _plain_quantize_case, "matmul": _plain_matmul}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return _EXACT[case["op"]](st)


def _exact_topk(st):
    V, k = st["case"]["V"], st["case"]["k"]
    parts = []
    for i in range(0, st["logits"].shape[0], 256):
        x = st["logits"][i:i + 256].double()
        d = torch.distributions.Categorical(logits=(x / TEMPERATURE).clamp_min(-1e300))
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
        pick = lambda ids: torch.log_softmax(x / TEMPERATURE, 1).gather(1, ids.long())     # noqa: E731
        parts.append([pick(st["tokens"][i:i + 256]), d.entropy(), torch.logsumexp(x / TEMPERATURE, 1),
                      order.to(torch.int32), pick(order)])
    out = [torch.cat(p) for p in zip(*parts)]
    if st["mask"] is not None:
        real = st["mask"].bool()
        for v, fill in zip(out, (0, 0, 0, -1, 0)):
            v[~real] = fill
    assert out[3].shape[1] == min(k, V)
    return dict(zip(("logprob", "entropy", "lse", "top_ids", "top_logprob"), out))


def _exact_topk_bwd(st):
    """By reverse mode through the library's log_softmax of the logits."""
    parts = []
    for i in range(0, st["logits"].shape[0], 256):
        part = slice(i, i + 256)
        x = st["logits"][part].double().requires_grad_(True)
        z = x / TEMPERATURE
        lp = torch.log_softmax(z, 1)
        h = -(lp.exp() * lp.masked_fill(lp == -math.inf, 0)).sum(1)
        total = ((lp.gather(1, st["tokens"][part].long()) * st["dlogprob"][part].double()).sum(1)
                 + (lp.gather(1, st["top_ids"][part].long()) * st["dtop"][part].double()).sum(1)
                 + h * st["dentropy"][part].double() + torch.logsumexp(z, 1) * st["dlse"][part].double())
        if st["mask"] is not None:
            total = total[st["mask"][part].bool()]
        parts.append(torch.autograd.grad(total.sum(), x)[0])
    return {"dlogits": torch.cat(parts)}


def _exact_quantize(st):
    """e4m3 by its grid: steps of 2^(e-3) in [2^e, 2^(e+1)), e >= -6, ties to even, largest 448."""
    block = st["case"]["block"]
    x = st["x"].t() if st["case"]["transpose"] else st["x"]
    R, C = x.shape
    q, s = [], []
    for i in range(0, R, 4096):                                       # (a multiple of 128 rows)
        part = x[i:i + 4096].double()
        up = torch.nn.functional.pad(part, (0, -C % 128, 0, -part.shape[0] % block))
        blocks = up.unflatten(0, (-1, block)).unflatten(2, (-1, 128))
        scale = blocks.abs().flatten(3).amax((1, 3)).clamp_min(MIN_AMAX) / E4M3_MAX
        v = blocks / scale[:, None, :, None]
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
        v = (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)
        q.append(v.flatten(2, 3).flatten(0, 1)[:part.shape[0], :C])
        s.append(scale)
    s = torch.cat(s)
    return {"q": torch.cat(q), "scales": s.t().contiguous() if block == 1 else s}


def _exact_matmul(st):
    a, b, sa, sb = st["a"].double(), st["b"].double(), st["a_scales"].double(), st["b_scales"].double()
    K, N = a.shape[1], b.shape[0]
    for kb in range(-(-K // 128)):                                    # block of the contraction by block
        cols = slice(kb * 128, min(K, kb * 128 + 128))
        if st["case"]["block"] == 1:
            scale_b = sb[kb]
        else:
            scale_b = sb[torch.arange(N, device=b.device) // 128, kb]
        a[:, cols] *= sa[kb][:, None]
        b[:, cols] *= scale_b[:, None]
    return a @ b.t()


_EXACT = {"topk": _exact_topk, "topk_bwd": _exact_topk_bwd, "quantize": _exact_quantize, "matmul": _exact_matmul}
