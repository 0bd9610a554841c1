"""CPU oracle for what surrounds the experts: the residual norm, its 8-bit rows and the router (numpy, fp64).

TEST INFRASTRUCTURE, NOT THE PRODUCT: only tests and the smoke check may import this module.  It shares nothing with the
CUDA library.  The formulas:

    h = x + r,  y = h / sqrt(mean(h^2) + eps) * w,  s = max |y| / 448 per group of columns,  q * s ~ y
    logit[t, e] = sum_h x[t, h] g[e, h] + b[e];  the k largest, equal ones lowest index first, never one at -inf;
    weight = exp(logit) / sum exp(logit) over the chosen experts, or over all of them
"""
import numpy as np


def add_rmsnorm(x, residual, weight, eps):
    """float64 arrays [rows, cols] (residual may be None), weight [cols].  Returns (h, y)."""
    h = x if residual is None else x + residual
    with np.errstate(all="ignore"):
        return h, h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps) * weight


def group_scales(y, group):
    """max |y| / 448 of every `group` columns (0: the whole row) -> [rows, groups]; NaN where the group has one."""
    rows, cols = y.shape
    group = cols if group <= 0 or group >= cols else group
    return np.stack([np.abs(y[:, a:a + group]).max(axis=1) for a in range(0, cols, group)], axis=1) / 448.0


def e4m3_to_f64(b):
    """The numbers that e4m3 bytes denote: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    b = np.asarray(b, dtype=np.uint8).astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    v = np.where((b & 0x7F) == 0x7F, np.nan, v)
    return np.where(b & 0x80, -v, v)


def choose(logits, k):
    """The choice alone, from logits [T, E] (float64, no NaN): ids [T, k], -1 where no expert above -inf is left."""
    ids = np.full((logits.shape[0], k), -1, np.int32)
    for t, row in enumerate(logits):
        order = sorted((e for e in range(row.size) if row[e] > -np.inf), key=lambda e: (-row[e], e))
        ids[t, :min(k, len(order))] = order[:k]
    return ids


def weights_of(logits, ids, renormalise=True):
    """Softmax weights of the chosen ids from logits [T, E] (float64)."""
    w = np.zeros(ids.shape)
    for t in range(ids.shape[0]):
        chosen = [e for e in ids[t] if e >= 0]
        if not chosen:
            continue
        top = max(logits[t, e] for e in chosen)
        over = chosen if renormalise else range(logits.shape[1])
        total = sum(np.exp(logits[t, e] - top) for e in over)
        w[t, :len(chosen)] = [np.exp(logits[t, e] - top) / total for e in chosen]
    return w
