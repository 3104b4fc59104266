"""Plain definitions of the block-scaled 8-bit operands and their product (test infrastructure; numpy only)."""
import numpy as np

MAX = 448.0
MIN_AMAX = 2.0 ** -100


def e4m3(v):
    """Nearest e4m3 value (ties to even, largest 448) of fp64 numbers: steps of 2^(e-3) in [2^e, 2^(e+1)), e >= -6."""
    v = np.asarray(v, np.float64)
    mag = np.maximum(np.abs(v), 2.0 ** -6)
    with np.errstate(invalid="ignore"):
        step = 2.0 ** (np.floor(np.log2(mag)) - 3)
        q = np.clip(np.round(v / step) * step, -MAX, MAX)
    return np.where(np.isnan(v), np.nan, q)


def _blocks(x, rows):
    R, C = x.shape
    for i, r in enumerate(range(0, R, rows)):
        for j, c in enumerate(range(0, C, 128)):
            yield i, j, slice(r, min(R, r + rows)), slice(c, min(C, c + 128))


def quantize(x, rows):
    """x [R, C] fp32 -> (q [R, C] as values, scales): the fp32 operations the definition names, each rounded once."""
    x = np.asarray(x, np.float32)
    R, C = x.shape
    kb = -(-C // 128)
    q = np.zeros((R, C))
    s = np.zeros((-(-R // rows), kb), np.float32)
    for i, j, r, c in _blocks(x, rows):
        a = np.abs(x[r, c]).max()
        if not np.isfinite(a):
            q[r, c], s[i, j] = np.nan, np.nan
            continue
        a = np.float32(max(float(a), MIN_AMAX))
        s[i, j] = a / np.float32(MAX)
        q[r, c] = e4m3((x[r, c] * (np.float32(MAX) / a)).astype(np.float64))
    return q, (np.ascontiguousarray(s.T) if rows == 1 else s)


def dequantize(q, s, rows):
    q = np.asarray(q, np.float64)
    R, C = q.shape
    s = np.asarray(s, np.float64)
    per_row = s.T if rows == 1 else np.repeat(s, 128, axis=0)[:R]
    return q * np.repeat(per_row, 128, axis=1)[:, :C]


def matmul(qa, sa, qb, sb, block_n):
    """(C, sum of absolute products) in fp64."""
    a, b = dequantize(qa, sa, 1), dequantize(qb, sb, block_n)
    return a @ b.T, np.abs(a) @ np.abs(b).T
