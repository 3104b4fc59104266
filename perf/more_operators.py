"""What the supervised fine-tuning operators of this library are measured on: the cases, their inputs, the operators in
plain torch operations, the library's own calls, and the same results in 64 bits.

  xent       ppo_lmhead_xent  cross entropy at the LM head, H [M,K] W [K,V], with both gradients and no [M,V] in memory
  embed      ppo_embed        rows of the embedding table, scaled
  embed_bwd  ppo_embed_bwd    gradient of the table: the rows' gradients summed per token
  clip       ppo_grad_clip    norm over many gradients and their clipping
"""
import math

import torch

own = False

IGNORE = -100          # label of a position that is not trained on
PAD = 1                # [PAD] token


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one response of 53 tokens: the two weight-sized matrices bound it
        {"name": "xent 53x50304x4096", "op": "xent", "M": 53, "K": 4096, "V": 50304, "layout": "kv", "T": 0,
         "ignored": 0.0, "shift": 0.0, "temperature": 1.0},
        # a batch of 64 responses x 53 tokens, padding after each response's end masked out
        {"name": "xent 3392x50304x4096 masked", "op": "xent", "M": 3392, "K": 4096, "V": 50304, "layout": "kv", "T": 53,
         "ignored": 0.0, "shift": 0.0, "temperature": 1.0},
        # a smaller model with the unpadded vocabulary, weight stored [V, K], prompt positions ignored by their label, all
        # logits far below 0 as some models have them
        {"name": "xent 1999x50277x1032 vk", "op": "xent", "M": 1999, "K": 1032, "V": 50277, "layout": "vk", "T": 0,
         "ignored": 0.3, "shift": -90.0, "temperature": 0.7},
        # the full batch of 512 responses x 53 tokens
        {"name": "xent 27136x50304x4096", "op": "xent", "M": 27136, "K": 4096, "V": 50304, "layout": "kv", "T": 0,
         "ignored": 0.0, "shift": 0.0, "temperature": 1.0},
        # the newest token of each of 53 sequences
        {"name": "embed 53x4096 bf16", "op": "embed", "N": 53, "K": 4096, "V": 50304, "dtype": "bf16", "out": "bf16",
         "scale": 1.0},
        # 512 sequences of 638 tokens (query and response)
        {"name": "embed 326656x4096 bf16", "op": "embed", "N": 326656, "K": 4096, "V": 50304, "dtype": "bf16",
         "out": "bf16", "scale": 64.0},
        # gradient of the table after one response: nearly all of it is zeros
        {"name": "embed_bwd 53x4096 bf16", "op": "embed_bwd", "N": 53, "K": 4096, "V": 50304, "dtype": "bf16",
         "out": "bf16", "pad": 0.0, "scale": 1.0},
        # rows at odd addresses, fp32 throughout, unpadded vocabulary
        {"name": "embed_bwd 5087x1021 fp32", "op": "embed_bwd", "N": 5087, "K": 1021, "V": 50277, "dtype": "fp32",
         "out": "fp32", "pad": 0.1, "scale": 32.0},
        # 512 responses x 53 tokens
        {"name": "embed_bwd 27136x4096 bf16", "op": "embed_bwd", "N": 27136, "K": 4096, "V": 50304, "dtype": "bf16",
         "out": "bf16", "pad": 0.3, "scale": 1.0},
        # 512 sequences of 638 tokens, fp32 gradient for the optimiser
        {"name": "embed_bwd 326656x4096 bf16 fp32", "op": "embed_bwd", "N": 326656, "K": 4096, "V": 50304,
         "dtype": "bf16", "out": "fp32", "pad": 0.3, "scale": 1.0},
        # a value head and the final norm
        {"name": "clip 4 small fp32", "op": "clip", "K": 4096, "V": 0, "layers": 0, "dtype": "fp32", "out": "fp32",
         "max_norm": 1.0, "scale": 1.0},
        # both vocabulary layers and four blocks of a model, clipped into fp32 for the optimiser
        {"name": "clip 50 bf16 fp32", "op": "clip", "K": 4096, "V": 50304, "layers": 4, "dtype": "bf16", "out": "fp32",
         "max_norm": 1.0, "scale": 0.125},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["xent", "xent", "embed", "embed_bwd", "clip"])
    dtype = rng.choice(["bf16", "fp32"])
    out = rng.choice(["bf16", "fp32"])
    if op == "xent":
        T = rng.choice([0, 53])
        M = _spread(rng, 1, 12000)
        if T:
            M = max(1, M // T) * T
        return {"op": op, "M": M, "K": 8 * _spread(rng, 8, 640), "V": rng.choice([50304, 50277, _spread(rng, 300, 60000)]),
                "layout": rng.choice(["kv", "vk"]), "T": T, "ignored": rng.choice([0.0, 0.0, 0.3]),
                "shift": rng.choice([0.0, 0.0, -90.0]), "temperature": rng.choice([1.0, 0.7])}
    if op in ("embed", "embed_bwd"):
        case = {"op": op, "N": _spread(rng, 1, 160000), "K": _spread(rng, 60, 4096),
                "V": rng.choice([50304, 50277, _spread(rng, 100, 60000)]), "dtype": dtype, "out": out,
                "scale": rng.choice([1.0, 1.0, 64.0])}
        if op == "embed_bwd":
            case["pad"] = rng.choice([0.0, 0.3])
        return case
    return {"op": op, "K": _spread(rng, 30, 3500), "V": rng.choice([0, 50277, 50304]), "layers": rng.randint(0, 4),
            "dtype": dtype, "out": out, "max_norm": rng.choice([1.0, 1e6]), "scale": rng.choice([1.0, 0.125])}


def _size(name):
    return 2 if name == "bf16" else 4


def work(case):
    op = case["op"]
    if op == "xent":
        M, K, V = case["M"], case["K"], case["V"]
        real = M * (0.5 * (1 + 1 / case["T"]) if case["T"] else 1.0) * (1 - case["ignored"])   # lengths are uniform in 1..T
        return {"bytes": 2 * (real * K + M * K + 2 * K * V) + 13 * M, "flops": 6 * real * K * V}
    if op == "clip":
        n = sum(math.prod(s) for s in _shapes(case))
        return {"bytes": n * (_size(case["dtype"]) + _size(case["out"])), "flops": 3 * n}
    N, K, V = case["N"], case["K"], case["V"]
    if op == "embed":
        seen = _distinct(N, V)
        return {"bytes": seen * K * _size(case["dtype"]) + N * (K * _size(case["out"]) + 4), "flops": N * K}
    real = N * (1 - case["pad"])
    return {"bytes": real * K * _size(case["dtype"]) + V * K * _size(case["out"]) + 4 * N, "flops": real * K}


def _distinct(N, V):
    """Expected number of different tokens among N of _tokens()."""
    span, step = math.log((V + 1) / 2), max(1, V // 2000)
    return min(V, sum(step * -math.expm1(N * math.log1p(-min(0.999, math.log1p(1 / (v + 2)) / span)))
                      for v in range(0, V, step)))


def _shapes(case):
    K, V = case["K"], case["V"]
    shapes = [(K, 1), (1,), (K,), (K,)]                                  # value head, final norm
    if V:
        shapes += [(V, K), (K, V)]                                       # embedding, LM head
    block = [(3 * K, K), (3 * K,), (K, K), (K,), (4 * K, K), (4 * K,), (K, 4 * K), (K,), (K,), (K,), (K,)]
    return shapes + block * case["layers"]


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _tokens(n, V, g):
    """Token ids whose frequency falls with the id, as those of text do."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return (2 * torch.exp(u * math.log((V + 1) / 2)) - 2).long().clamp(0, V - 1).to(torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    randn = lambda *s, **kw: torch.randn(*s, generator=g, device=dev, **kw)         # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=g, device=dev)                       # noqa: E731
    op = case["op"]
    st = {"case": dict(case)}
    if op == "xent":
        M, K, V = case["M"], case["K"], case["V"]
        shape, pitch = ((K, V), -(-V // 8) * 8) if case["layout"] == "kv" else ((V, K), K)
        w = torch.zeros((shape[0], pitch), dtype=torch.bfloat16, device=dev)        # rows of 16-byte multiples
        w[:, :shape[1]] = randn(*shape) * (3.0 / math.sqrt(K))                      # logits of +-3 and more
        w = w[:, :shape[1]]
        st["W"] = w if case["layout"] == "kv" else w.t()                            # [K, V]
        st["W"][0] = case["shift"] / 8                                              # all logits of a row lie about there
        st["labels"] = _tokens(M, V, g)
        h = randn(M, K) * (0.5 + rand(M, 1))
        # the model has learnt something: a part of each state points at its label
        h += 1.3 * rand(M, 1) * st["W"][:, st["labels"].long()].t().float()
        h[:, 0] = 8
        st["H"] = h.to(torch.bfloat16)
        st["labels"][rand(M) < case["ignored"]] = IGNORE
        st["mask"] = None
        if case["T"]:
            length = torch.randint(1, case["T"] + 1, (M // case["T"], 1), generator=g, device=dev) if M >= case["T"] else \
                torch.ones((M, 1), device=dev)
            st["mask"] = (torch.arange(M // length.shape[0], device=dev)[None] < length).to(torch.uint8).reshape(M)
        return st
    if op == "clip":
        st["grads"] = []
        for i, shape in enumerate(_shapes(case)):
            x = randn(*shape, dtype=_dtype(case["dtype"]))
            st["grads"].append(x.mul_(0.01 * (1 + i % 5)))
        st["out"] = [torch.empty_like(x, dtype=_dtype(case["out"])) for x in st["grads"]]
        return st
    N, K, V = case["N"], case["K"], case["V"]
    st["tokens"] = _tokens(N, V, g)
    if op == "embed":
        st["table"] = randn(V, K, dtype=_dtype(case["dtype"])) * 0.02
    else:
        st["tokens"][rand(N) < case["pad"]] = PAD
        st["dY"] = randn(N, K, dtype=_dtype(case["dtype"])) * 1e-3
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    op = st["case"]["op"]
    if own:
        return _OWN[op](st)
    return _PLAIN[op](st)


def _own_xent(st):
    from paper_2403_17031_b200 import binding as b
    return b.lmhead_xent(st["H"], st["W"], st["labels"], mask=st["mask"], ignore_id=IGNORE,
                         temperature=st["case"]["temperature"])


def _own_embed(st):
    from paper_2403_17031_b200 import binding as b
    return b.embed(st["table"], st["tokens"], scale=st["case"]["scale"], out_dtype=_dtype(st["case"]["out"]))


def _own_embed_bwd(st):
    from paper_2403_17031_b200 import binding as b
    return b.embed_bwd(st["dY"], st["tokens"], st["case"]["V"], scale=st["case"]["scale"], padding_id=PAD,
                       out_dtype=_dtype(st["case"]["out"]))


def _own_clip(st):
    from paper_2403_17031_b200 import binding as b
    norm = b.grad_clip(st["grads"], st["case"]["max_norm"], scale=st["case"]["scale"], out=st["out"])
    return {"grads": st["out"], "norm": norm}


# ---- the plain forms
def _plain_xent(st):
    tau, M = st["case"]["temperature"], st["H"].shape[0]
    h, w, labels = st["H"].float(), st["W"].float(), st["labels"].long()
    real = labels != IGNORE
    if st["mask"] is not None:
        real &= st["mask"] != 0
    rows = real.nonzero()[:, 0]
    h, labels, n = h[rows], labels[rows], rows.numel()
    z = h @ w
    z /= tau
    top = z.max(1, keepdim=True).values if n else z.sum(1, keepdim=True)
    picked = z.gather(1, labels[:, None])[:, 0]
    z -= top
    z.exp_()
    s = z.sum(1, keepdim=True)
    lse = (top + torch.log(s))[:, 0]
    nll = lse - picked
    z /= s                                                               # from here on softmax, then the gradient
    z[torch.arange(n, device=z.device), labels] -= 1
    z *= 1.0 / (max(n, 1) * tau)
    full = lambda v: torch.zeros((M, *v.shape[1:]), dtype=v.dtype, device=v.device).index_copy_(0, rows, v)   # noqa: E731
    dw = (h.t() @ z).to(torch.bfloat16) if st["W"].stride(1) == 1 else (z.t() @ h).to(torch.bfloat16).t()
    return {"loss": nll.sum() / max(n, 1), "nll": full(nll), "lse": full(lse), "dH": full((z @ w.t()).to(torch.bfloat16)),
            "dW": dw}


def _plain_embed(st):
    return (st["table"][st["tokens"].long()].float() * st["case"]["scale"]).to(_dtype(st["case"]["out"]))


def _plain_embed_bwd(st):
    tokens, K = st["tokens"].long(), st["dY"].shape[1]
    d = torch.zeros((st["case"]["V"], K), dtype=torch.float32, device=tokens.device)
    rows = (tokens != PAD).nonzero()[:, 0]
    d.index_add_(0, tokens[rows], st["dY"][rows].float())
    d *= st["case"]["scale"]
    return d.to(_dtype(st["case"]["out"]))


def _plain_clip(st):
    case = st["case"]
    squares = torch.stack([x.float().square().sum(dtype=torch.float64) for x in st["grads"]]).sum()
    norm = torch.sqrt(squares) * abs(case["scale"])
    coef = torch.where(norm > case["max_norm"], case["max_norm"] / norm, torch.ones_like(norm))
    factor = (coef * case["scale"]).float()
    return {"grads": [(x.float() * factor).to(_dtype(case["out"])) for x in st["grads"]],
            "norm": torch.stack([norm, coef]).float()}


_OWN = {"xent": _own_xent, "embed": _own_embed, "embed_bwd": _own_embed_bwd, "clip": _own_clip}
_PLAIN = {"xent": _plain_xent, "embed": _plain_embed, "embed_bwd": _plain_embed_bwd, "clip": _plain_clip}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return _EXACT[case["op"]](st)


def _exact_xent(st):
    """By reverse mode through the library's cross entropy, some rows at a time."""
    labels = st["labels"].long()
    if st["mask"] is not None:
        labels = labels.masked_fill(st["mask"] == 0, IGNORE)
    n = max(1, int((labels != IGNORE).sum()))
    w = st["W"].double().requires_grad_(True)
    lse, nll, dh = [], [], []
    for i in range(0, labels.shape[0], 2048):
        h = st["H"][i:i + 2048].double().requires_grad_(True)
        z = (h @ w) / st["case"]["temperature"]
        lab = labels[i:i + 2048]
        loss = torch.nn.functional.cross_entropy(z, lab, ignore_index=IGNORE, reduction="none")
        (loss.sum() / n).backward()
        nll.append(loss.detach())
        lse.append(torch.logsumexp(z.detach(), 1).masked_fill(lab == IGNORE, 0))
        dh.append(h.grad)
    nll = torch.cat(nll)
    return {"loss": nll.sum() / n, "nll": nll, "lse": torch.cat(lse), "dH": torch.cat(dh), "dW": w.grad}


def _exact_embed(st):
    return torch.nn.functional.embedding(st["tokens"].long(), st["table"]).double() * st["case"]["scale"]


def _exact_embed_bwd(st):
    """Column by column of the one-hot product, a few columns at a time."""
    tokens, V = st["tokens"].long(), st["case"]["V"]
    parts = []
    for cols in st["dY"].split(256, 1):
        d = torch.zeros((V, cols.shape[1]), dtype=torch.float64, device=cols.device)
        d.scatter_add_(0, tokens[:, None].expand(-1, cols.shape[1]), cols.double())
        d[PAD] = 0
        parts.append(d * st["case"]["scale"])
    return torch.cat(parts, 1)


def _exact_clip(st):
    case = st["case"]
    norm = abs(case["scale"]) * math.sqrt(sum(float(torch.linalg.vector_norm(x.double())) ** 2 for x in st["grads"]))
    coef = min(1.0, case["max_norm"] / norm)
    return {"grads": [x.double() * (case["scale"] * coef) for x in st["grads"]],
            "norm": torch.tensor([norm, coef], dtype=torch.float64)}


_EXACT = {"xent": _exact_xent, "embed": _exact_embed, "embed_bwd": _exact_embed_bwd, "clip": _exact_clip}
