"""The operators at the output end of a language model in 64 bits, from their definitions: norm with the
residual's addition and its gradients, the scaled integer product, sampling, distillation.  Plain numpy, no code of the library."""
from __future__ import annotations

import math

import numpy as np


def rms_norm(x, weight, eps, residual=None):
    """(y, h, rms) with h = x + residual, y = weight h / rms, all FP64."""
    h = x.astype(np.float64) + (0.0 if residual is None else residual.astype(np.float64))
    rms = np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    w = 1.0 if weight is None else weight.astype(np.float64)
    return w * h / rms, h, rms


def rows_in_8_bits(h32, weight, most):
    """(quotients p (most (1 / m)) before rounding, m = largest |p| = |w h| of the rows): h32 is the FP32 stream the norm's rows are taken from."""
    p = h32.astype(np.float64) * (1.0 if weight is None else weight.astype(np.float64))
    m = np.max(np.abs(p), axis=1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        return np.where(m > 0, p * (1.0 / m * most), 0.0), m


def rms_norm_backward(dy, h, weight, eps, dsum=None):
    """(dh, dweight), by the quotient rule."""
    dy, h = dy.astype(np.float64), h.astype(np.float64)
    d = h.shape[1]
    rms = np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    g = dy * (1.0 if weight is None else weight.astype(np.float64))
    dh = g / rms - h * np.sum(g * h, axis=1, keepdims=True) / (d * rms ** 3)
    if dsum is not None:
        dh = dh + dsum.astype(np.float64)
    return dh, np.sum(dy * h / rms, axis=0)


def int8_matmul(a, a_scale, b, b_scale, bias=None):
    acc = a.astype(np.int64) @ b.astype(np.int64).T
    out = acc * a_scale.astype(np.float64)[:, None] * b_scale.astype(np.float64)[None, :]
    return out if bias is None else out + bias.astype(np.float64)


def sample_row(z, u, t=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Kept tokens in order of index, their weights' running sum, and the place u falls on: (index, cumulative, token, kept share).
    token = -1 where nothing can be drawn."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    if not np.any(z > -np.inf):
        return np.zeros(0, np.int64), np.zeros(0), -1, 0.0
    if not t > 0:
        t, top_k = 1.0, 1
    order = np.argsort(-z, kind="stable")
    order = order[z[order] > -np.inf]
    if 0 < top_k < len(order):
        order = order[:top_k]
    top = z[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(z[order] == top, 1.0, np.exp((z[order] - top) / t))
    n = len(order)
    if top_p < 1:
        c = np.cumsum(w)
        n = max(1, int(np.searchsorted(c, top_p * c[-1])) + 1)
        n = min(n, len(order))
    if min_p > 0:
        n = min(n, int(np.count_nonzero(w >= min(min_p, 1.0))))
    kept = np.argsort(order[:n])
    index, w = order[:n][kept], w[:n][kept]
    c = np.cumsum(w)
    u = 0.0 if not u > 0 else min(u, 1.0)
    j = min(int(np.searchsorted(c, u * c[-1], side="right")), len(w) - 1)
    while w[j] == 0.0:
        j -= 1
    return index, c, int(index[j]), w[j] / c[-1]


def distill(z, teacher_idx, teacher_logits, T, weight=None):
    """(loss, gradient) row by row; entries outside [0, V) do not count."""
    rows, V = z.shape
    loss, grad = np.zeros(rows), np.zeros((rows, V))
    for r in range(rows):
        v = 1.0 if weight is None else float(weight[r])
        ok = (teacher_idx[r] >= 0) & (teacher_idx[r] < V)
        at, t = teacher_idx[r][ok], teacher_logits[r][ok].astype(np.float64) / T
        if v == 0.0 or not np.any(t > -np.inf):
            continue
        q = np.exp(t - t.max())
        logq = t - t.max() - math.log(q.sum())
        q /= q.sum()
        s = z[r].astype(np.float64) / T
        if not np.any(s > -np.inf):
            p, logp = np.zeros(V), np.full(V, -np.inf)
        else:
            e = np.exp(s - s.max())
            p, logp = e / e.sum(), s - s.max() - math.log(e.sum())
        there = q > 0
        loss[r] = v * T * T * np.sum(q[there] * (logq[there] - logp[at[there]]))
        grad[r] = p
        np.subtract.at(grad[r], at, q)
        grad[r] *= v * T
    return loss, grad
