"""Plain fp64 definitions of the supervised fine-tuning calls (test infrastructure; numpy only)."""
import numpy as np


def xent(H, W, labels, real, tau, scale=1.0, denom=None):
    """H [M, K], W [K, V] -> dict(loss, nll, lse, dH, dW, D) over the rows with real != 0; D is the gradient on the logits."""
    H, W = np.asarray(H, np.float64), np.asarray(W, np.float64)
    tau, real = np.float64(np.float32(tau)), np.asarray(real) != 0
    M, V = H.shape[0], W.shape[1]
    nll, lse, D = np.zeros(M), np.zeros(M), np.zeros((M, V))
    n = int(real.sum())
    d = np.float64(denom) if denom is not None else max(n, 1)
    for r in np.flatnonzero(real):
        z = H[r] @ W / tau
        m = z.max()
        e = np.exp(z - m)
        lse[r] = m + np.log(e.sum())
        D[r] = np.float64(np.float32(scale)) / (d * tau) * e / e.sum()
        if 0 <= labels[r] < V:
            nll[r] = lse[r] - z[labels[r]]
            rest = np.delete(e, labels[r]).sum()                     # 1 - p without cancellation
            D[r, labels[r]] = -np.float64(np.float32(scale)) / (d * tau) * rest / e.sum()
        else:
            nll[r], D[r] = np.nan, np.nan
    return {"loss": nll.sum() / d if n else 0.0, "nll": nll, "lse": lse, "dH": D @ W.T, "dW": H[real].T @ D[real], "D": D}


def embed(table, tokens, scale):
    table, tokens = np.asarray(table, np.float64), np.asarray(tokens)
    out = np.full((tokens.size, table.shape[1]), np.nan)
    ok = (tokens >= 0) & (tokens < table.shape[0])
    out[ok] = table[tokens[ok]] * np.float64(np.float32(scale))
    return out


def embed_bwd(dY, tokens, V, scale, padding_id=-1, base=None):
    """(gradient of the table, the same sums over absolute values: the scale errors are measured on)."""
    dY = np.asarray(dY, np.float64)
    d, size = np.zeros((V, dY.shape[1])), np.zeros((V, dY.shape[1]))
    for i, t in enumerate(np.asarray(tokens)):
        if 0 <= t < V and t != padding_id:
            d[t] += dY[i]
            size[t] += np.abs(dY[i])
    s = np.float64(np.float32(scale))
    d, size = d * s, size * abs(s)
    return (d if base is None else d + np.asarray(base, np.float64)), size


def grad_clip(grads, max_norm, scale):
    """(scaled gradients, norm, factor)."""
    s, most = np.float64(np.float32(scale)), np.float64(np.float32(max_norm))
    norm = abs(s) * np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads))
    coef = most / norm if norm > most else 1.0
    return [np.asarray(g, np.float64) * (s * coef) for g in grads], norm, coef
