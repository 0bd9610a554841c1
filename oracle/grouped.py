"""CPU oracle for the grouped products, the lists they go by, and 8-bit rows (numpy, fp64).

TEST INFRASTRUCTURE, NOT THE PRODUCT: only tests and the smoke check may import this module.  It shares nothing with the
CUDA library.  The formulas:

    rows of the product: the choices in ascending order of (expert, choice); place = the row of each choice, -1 for none
    out[r, n] = sum_c x[src(r), c] W_e[n, c]   (a pair: silu(first) * second)
    out[t] = sum_j w[t, j] y[place[t, j]]
    a = max |x|,  q = rint(127 x / a),  scale = a / 127
"""
import numpy as np

from oracle.ffn import silu


def group(ids, n_experts):
    """ids [T, k] -> offsets [n_experts + 1], order (of the choices that have an expert), place [T, k]."""
    flat = np.asarray(ids).ravel()
    order, offsets = [], [0]
    for e in range(n_experts):
        order += [c for c in range(flat.size) if flat[c] == e] if flat.size < 4096 else np.nonzero(flat == e)[0].tolist()
        offsets.append(len(order))
    place = np.full(flat.size, -1, np.int64)
    place[np.asarray(order, np.int64)] = np.arange(len(order))
    return np.array(offsets), np.array(order, np.int64), place.reshape(np.shape(ids))


def products(x, src, offsets, matrices):
    """x [*, cols], src [rows]: row of x per row of the product -> [offsets[-1], rows of the matrices], float64."""
    out = np.zeros((int(offsets[-1]), matrices[0].shape[0]))
    for e, w in enumerate(matrices):
        rows = slice(int(offsets[e]), int(offsets[e + 1]))
        out[rows] = x[src[rows]] @ w.T
    return out


def gated(first, second):
    return silu(first) * second


def combine(y, place, weights):
    """y [rows, cols], place [T, k], weights [T, k] or None -> [T, cols]."""
    out = np.zeros((place.shape[0], y.shape[1]))
    for t in range(place.shape[0]):
        for j in range(place.shape[1]):
            if place[t, j] >= 0:
                out[t] += (1.0 if weights is None else weights[t, j]) * y[place[t, j]]
    return out


def quantize(x):
    """x [rows, cols] float64 -> q (int64), scales."""
    with np.errstate(all="ignore"):
        a = np.abs(x).max(axis=1)
        fine = np.isfinite(a)
        q = np.where((fine & (a > 0))[:, None], np.rint(np.nan_to_num(x * 127 / a[:, None])), 0)
    return q.astype(np.int64), np.where(fine, a / 127, np.nan)
