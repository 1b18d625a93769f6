"""64-bit references of the operators around the linears, in numpy, from their definitions."""
import math

import numpy as np

SCALE_NONE, SCALE_LINEAR, SCALE_BY_TURNS, SCALE_BY_INDEX = range(4)


def norm(v, layer, eps, factor=1.0, bias=0.0):
    """Rows of v normalised; also the sizes that errors go by: |v - mean| / sqrt(..) and its factor."""
    c = v - v.mean(-1, keepdims=True) if layer else v
    return c / np.sqrt((c * c).mean(-1, keepdims=True) + eps) * factor + bias


def frequency(rot, i, base, scaling=SCALE_NONE, factor=1.0, trained=0, low=1.0, high=32.0):
    theta = base ** (-2.0 * i / rot)
    if scaling == SCALE_NONE:
        return theta
    if scaling == SCALE_LINEAR:
        return theta / factor
    if scaling == SCALE_BY_TURNS:
        kept = (trained * theta / math.tau - low) / (high - low)
    else:
        at = [rot / 2 * math.log(trained / (math.tau * n)) / math.log(base) for n in (high, low)]
        first, last = max(0, math.floor(at[0])), min(rot - 1, math.ceil(at[1]))
        kept = 1 - (i - first) / max(last - first, 0.001)
    kept = min(1.0, max(0.0, kept))
    return theta * kept + theta / factor * (1 - kept)


def rotate(heads, positions, theta, pairs, factor=1.0):
    """heads [rows, n, d] turned by positions [rows] in their first 2 len(theta) values."""
    out = heads.astype(np.float64).copy()
    half = len(theta)
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(theta)
    c, s = np.cos(angle) * factor, np.sin(angle) * factor
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    a, b = out[..., first].copy(), out[..., second].copy()
    out[..., first] = a * c - b * s
    out[..., second] = a * s + b * c
    return out


def order(x):
    """Whole numbers in the order of x: totalOrder, every NaN below all numbers."""
    bits = np.ascontiguousarray(x, dtype=np.float32).view(np.int32).astype(np.int64)
    key = np.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    return np.where(np.isnan(x), -2 ** 40, key)


def top(x, k):
    """Columns of the k largest of each row, descending, equal ones by column."""
    return np.argsort(-order(x), axis=-1, kind="stable")[:, :k]


def log_probs(x):
    """Log probabilities and entropy of rows of logits."""
    x = x.astype(np.float64)
    lp, h = np.empty_like(x), np.empty(len(x))
    for i, row in enumerate(x):
        if np.isnan(row).any() or (row == np.inf).any():
            lp[i], h[i] = np.nan, np.nan
        elif (row == -np.inf).all():
            lp[i], h[i] = -np.inf, 0.0
        else:
            z = row - row.max()
            lp[i] = z - np.log(np.exp(z).sum())
            p = np.exp(lp[i])
            h[i] = -(p * np.where(p > 0, lp[i], 0.0)).sum()
    return lp, h


def adapters(x, base, A, B, scale, ids):
    """ids: each row's adapter, -1 for none.  Also the sizes that errors go by."""
    out, size = base.astype(np.float64).copy(), np.zeros(base.shape)
    for m, a in enumerate(ids):
        if a >= 0:
            t = scale[a] * (A[a].astype(np.float64) @ x[m])
            out[m] += B[a].astype(np.float64) @ t
            size[m] = np.abs(B[a]).astype(np.float64) @ (np.abs(scale[a]) * (np.abs(A[a]).astype(np.float64) @ np.abs(x[m])))
    return out, size
