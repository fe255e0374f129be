"""The operators around a language model's tokens, in 64 bits -- TEST
INFRASTRUCTURE ONLY.  Plain numpy from the operators' definitions (lda_draw.h);
shares nothing with the kernels but the generator's definition."""
from __future__ import annotations

import numpy as np

from .philox import philox4x32_np

GROUP = 1024


def keep_factor(rows: int, cols: int, p: float, seed: int, step: int) -> np.ndarray:
    """float64 [rows][cols]: 0 where dropped, else 1 / P(kept)."""
    q = min(65535, int(np.rint(65536.0 * p)))
    groups = (cols + 7) // 8
    words = philox4x32_np(np.arange(groups)[None, :], np.arange(rows)[:, None], step, 1,
                          seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    half = np.zeros((rows, groups, 8), dtype=np.int64)
    for j, w in enumerate(words):
        half[:, :, 2 * j] = w & np.uint32(0xFFFF)
        half[:, :, 2 * j + 1] = w >> np.uint32(16)
    keep = half.reshape(rows, groups * 8)[:, :cols] >= q
    return keep * (65536.0 / (65536 - q))


def dropout(x, p, seed, step):
    """x float64 [rows][cols]."""
    f = keep_factor(x.shape[0], x.shape[1], p, seed, step)
    return np.where(f > 0, x, 0.0) * f


def embed(table, word_id, scale, p=0.0, seed=0, step=0):
    V = table.shape[0]
    ok = (word_id >= 0) & (word_id < V)
    x = np.where(ok[:, None], table[np.clip(word_id, 0, V - 1)] * scale, 0.0)
    return dropout(x, p, seed, step) if p else x


def embed_grad(grad, word_id, V, scale, p=0.0, seed=0, step=0):
    """(gradient [V][D], sum of the terms' magnitudes [V][D], tokens [V])."""
    N, D = grad.shape
    x = (dropout(grad, p, seed, step) if p else grad) * scale
    ok = (word_id >= 0) & (word_id < V)
    out, size = np.zeros((V, D)), np.zeros((V, D))
    np.add.at(out, word_id[ok], x[ok])
    np.add.at(size, word_id[ok], np.abs(x[ok]))
    return out, size, np.bincount(word_id[ok], minlength=V)


def penalise(x, history=None, lengths=None, prompt=None, repetition=None, frequency=None,
             presence=None, bias=None, mask=None):
    """(logits float64 [B][V] under the rules, the largest magnitude met on the
    way [B][V]).  mask: truth values [B][V] or [V]."""
    x = np.array(x, dtype=np.float64)
    B, V = x.shape
    size = np.abs(x)
    if history is not None:
        for b in range(B):
            n = max(0, min(int(lengths[b]), history.shape[1]))
            first = int(prompt[b]) if prompt is not None else 0
            h = history[b, :n]
            made = h[max(0, first):]
            seen = np.bincount(h[(h >= 0) & (h < V)], minlength=V) > 0
            c = np.bincount(made[(made >= 0) & (made < V)], minlength=V)
            r = float(repetition[b]) if repetition is not None else 1.0
            f = float(frequency[b]) if frequency is not None else 0.0
            p = float(presence[b]) if presence is not None else 0.0
            x[b] = np.where(seen, np.where(x[b] > 0, x[b] / r, x[b] * r), x[b])
            size[b] = np.maximum(size[b], np.abs(x[b])) + abs(f) * c + abs(p)
            x[b] = x[b] - f * c - p * (c > 0)
    if bias is not None:
        x = x + bias
        size = size + np.where(np.isfinite(bias), np.abs(bias), 0.0)
    if mask is not None:
        x = np.where(mask, x, -np.inf)
    return x, size


def mask_words(allowed: np.ndarray) -> np.ndarray:
    """Truth values [..., V] as int32 words [..., ceil(V / 32)]."""
    V = allowed.shape[-1]
    pad = np.zeros(allowed.shape[:-1] + ((V + 31) // 32 * 32,), dtype=np.uint8)
    pad[..., :V] = allowed
    return np.packbits(pad, axis=-1, bitorder="little").view(np.int32)


def _uniforms(index, position, domain, seed):
    y = philox4x32_np(np.asarray(index), int(position) & 0xFFFFFFFF, 0, domain,
                      int(seed) & 0xFFFFFFFF, (int(seed) >> 32) & 0xFFFFFFFF)[0]
    return (y.astype(np.float64) + 0.5) * 2.0 ** -32


def _race(u, w):
    """(winner, how much the second best key is above it, relatively): keys
    -log(1 - u) / w.  A key is blurred by the fp32 rounding of u, which matters
    where u is next to 1."""
    with np.errstate(divide="ignore", invalid="ignore"):
        e = -np.log1p(-u)
        key = np.where(w > 0, e / w, np.inf)
        blur = 1 + 2.0 ** -23 / ((1 - u) * e)
    best = int(np.argmin(key))
    rest = np.delete(key / blur, best)
    second = rest.min() if rest.size else np.inf
    return best, second / (key[best] * blur[best]) - 1


def draw(x, temperature, min_p, seed, position):
    """One row of logits (float64, the rules applied): (token, probability,
    margin), the margin by which the winning keys are the smallest and the floor
    does not decide."""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return -1, 0.0, np.inf
    if not temperature > 0:
        return int(np.argmax(x)), 1.0, np.inf
    if np.isposinf(top):
        w = (x == top).astype(np.float64)
    else:
        w = np.exp((x - top) / min(temperature, 1e30))
    margin = np.inf
    if min_p > 0:
        floor = min(min_p, 1.0)
        near = w[(w != 1.0) & (w > 0)]
        margin = np.abs(near / floor - 1).min() if near.size else np.inf
        w = np.where(w >= floor, w, 0.0)
    starts = np.arange(0, len(w), GROUP)
    mass = np.add.reduceat(w, starts)
    g, m = _race(_uniforms(np.arange(len(starts)), position, 2, seed), mass)
    at = np.arange(g * GROUP, min(len(w), (g + 1) * GROUP))
    i, n = _race(_uniforms(at, position, 3, seed), w[at])
    return int(at[i]), w[at[i]] / w.sum(), min(margin, m, n)
