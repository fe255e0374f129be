"""The operators between a layer's last activations and the next token, in 64 bits
-- TEST INFRASTRUCTURE ONLY.  Plain numpy from the operators' definitions
(lda_draw.h)."""
from __future__ import annotations

import numpy as np


def norm(x, weight, eps, residual=None):
    """(y, h), float64 [N][D]."""
    h = x if residual is None else x + residual
    return h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * weight, h


def norm_grad(grad, h, weight, eps, residual=None):
    """(dx, dweight, what the terms of dx add up to without their signs, the same of
    dweight)."""
    s = 1 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    v, d = h * s, grad * weight
    along = (d * v).mean(1, keepdims=True)
    r = 0.0 if residual is None else residual
    size = np.abs(s * d) + np.abs(s * v) * np.abs(d * v).mean(1, keepdims=True) + np.abs(r)
    return s * (d - v * along) + r, (grad * v).sum(0), size, np.abs(grad * v).sum(0)


def quantise(x):
    """(q before it is rounded, scale) of each row; NaN scales and zeros where a row is
    not finite."""
    top = np.abs(x).max(1)
    fine = np.isfinite(top)
    at = np.where(fine & (top > 0), top, 1.0)[:, None]
    q = np.where(fine[:, None], 127.0 * np.where(fine[:, None], x, 0.0) / at, 0.0)
    return q, np.where(fine, top / 127, np.nan)


def project(q, scale, weight, weight_scale, bias=None):
    """(out, the product without the bias): the sums of whole numbers are exact in 64
    bits."""
    y = (q.astype(np.float64) @ weight.astype(np.float64).T) * scale[:, None] * weight_scale
    return (y if bias is None else y + bias), y


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row of logits (float64): (token, probability, margin), the margin by which sums
    of weights decide, relative to the largest weight."""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return -1, 0.0, np.inf
    if not temperature > 0:
        return int(np.argmax(x)), 1.0, np.inf
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.exp((x - top) / temperature)
    w = np.where(x == top, 1.0, np.where(np.isneginf(x) | np.isposinf(top), 0.0, w))
    margin = np.inf
    order = np.argsort(-x, kind="stable")
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        sums = np.cumsum(w[order])
        at = max(top_p, 0.0) * sums[-1]
        n = max(0, int(np.searchsorted(sums, at)))
        near = np.abs(sums - at)
        margin = near[near > 0].min(initial=np.inf)
        order = order[:n + 1]
    if min_p > 0:
        floor = min(min_p, 1.0)
        near = w[order][(w[order] != 1.0) & (w[order] > 0)]
        margin = min(margin, np.abs(near - floor).min(initial=np.inf))
        order = order[w[order] >= floor]
    stay = np.sort(order)
    sums = np.cumsum(w[stay])
    at = (u if u > 0 else 0.0) * sums[-1]
    i = int(np.searchsorted(sums, at, side="right"))
    if i >= len(stay):  # u of 1 and above: the last with a weight
        i = int(np.nonzero(w[stay])[0][-1])
    else:
        margin = min(margin, np.abs(sums - at).min() if at > 0 else np.inf)
    return int(stay[i]), w[stay[i]] / sums[-1], margin
