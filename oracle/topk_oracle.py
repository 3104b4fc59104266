"""Plain fp64 definition of the alternatives call and its gradient (test infrastructure; numpy only)."""
import numpy as np

NO_WEIGHT = -1e30      # a logit at or below this has probability 0


def topk(x, tokens, k, tau, mask=None):
    """x [rows, V] (the stored logits, exactly), tokens [rows, n] -> dict like the library's; rows without a distribution
    (NaN, +inf, no logit with weight) are NaN with ids -1, masked rows 0 with ids -1."""
    x = np.asarray(x, np.float64)
    rows, V = x.shape
    n = tokens.shape[1]
    out = {"logprob": np.zeros((rows, n)), "entropy": np.zeros(rows), "lse": np.zeros(rows),
           "top_ids": np.full((rows, k), -1, np.int32), "top_logprob": np.zeros((rows, k))}
    for r in range(rows):
        if mask is not None and not mask[r]:
            continue
        row = x[r]
        z = row / np.float64(tau)
        live = row > NO_WEIGHT
        if np.isnan(row).any() or np.isposinf(row).any() or not live.any():
            for name in ("logprob", "entropy", "lse", "top_logprob"):
                out[name][r] = np.nan
            continue
        m = z[live].max()
        e = np.exp(z[live] - m)
        lse = m + np.log(e.sum())
        lp = z[live] - lse
        out["lse"][r] = lse
        out["entropy"][r] = -(np.exp(lp) * lp).sum()
        order = np.argsort(-row, kind="stable")[:k]
        out["top_ids"][r] = order
        out["top_logprob"][r] = z[order] - lse
        for i, t in enumerate(tokens[r]):
            out["logprob"][r, i] = z[t] - lse if 0 <= t < V else np.nan
    return out


def topk_bwd(x, ids, g, lse, tau, entropy=None, dentropy=None, dlse=None, mask=None):
    """Gradient on the logits [rows, V], and the same sum over absolute values (the scale errors are measured on)."""
    x = np.asarray(x, np.float64)
    rows, V = x.shape
    d, size = np.zeros((rows, V)), np.zeros((rows, V))
    for r in range(rows):
        if mask is not None and not mask[r]:
            continue
        if ids.shape[1] and ((ids[r] < 0) | (ids[r] >= V)).any():
            d[r] = np.nan
            continue
        lp = x[r] / np.float64(tau) - np.float64(lse[r])
        p = np.exp(lp)
        lp = np.where(p > 0, lp, 0.0)
        h = 0.0 if dentropy is None else np.float64(dentropy[r])
        H = 0.0 if dentropy is None else np.float64(entropy[r])
        a = 0.0 if dlse is None else np.float64(dlse[r])
        G = g[r].astype(np.float64).sum()
        d[r] = p * (a - G - h * (lp + H))
        size[r] = p * (abs(a) + np.abs(g[r]).sum() + abs(h) * (np.abs(lp) + abs(H)))
        np.add.at(d[r], ids[r], g[r].astype(np.float64))
        np.add.at(size[r], ids[r], np.abs(g[r]).astype(np.float64))
    return d / np.float64(tau), size / np.float64(tau)
