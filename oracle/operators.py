"""CPU oracle of the operators around the synchronization, in 64 bits.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain numpy, written
from the formulas, nothing imported from the product.

  lookup          out[t] = scale * table[ids[t]], zeros for an id outside the table
  embedding_grad  grad[r] = scale * sum of dout[t] over the tokens of row r
  grad_norm       the 2-norm over a list of gradients
  adamw           one AdamW step on one tensor
  held_first, held_second, nearest_first, nearest_second
                  the 8-bit codes of the two moments: what a code stands for, and
                  the nearest code of a value in the root's scale
"""
from __future__ import annotations

import numpy as np

BLOCK = 256        # elements of an 8-bit state that share a scale


def lookup(table: np.ndarray, ids: np.ndarray, scale: float) -> np.ndarray:
    out = np.zeros((len(ids), table.shape[1]))
    for t, r in enumerate(ids):
        if 0 <= r < len(table):
            out[t] = scale * table[r].astype(np.float64)
    return out


def embedding_grad(rows: int, ids: np.ndarray, dout: np.ndarray, scale: float, padding: int = -1,
                   old: np.ndarray | None = None):
    """(grad, magnitude): magnitude[r] = sum of |scale * dout[t]| (and |old|), the scale of rounding errors."""
    grad = np.zeros((rows, dout.shape[1]))
    magnitude = np.zeros_like(grad)
    for t, r in enumerate(ids):
        if 0 <= r < rows and r != padding:
            grad[r] += scale * dout[t].astype(np.float64)
            magnitude[r] += np.abs(scale * dout[t].astype(np.float64))
    if old is not None:
        grad += old
        magnitude += np.abs(old)
    return grad, magnitude


def grad_norm(grads) -> float:
    return float(np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads)))


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, decay, grad_scale=1.0, max_norm=0.0, norm=0.0):
    """(p, m, v) after step number t; norm is that of the unscaled gradients."""
    p, g, m, v = (x.astype(np.float64) for x in (p, g, m, v))
    g = g * grad_scale
    if max_norm > 0.0:
        g = g * np.minimum(1.0, max_norm / (abs(grad_scale) * norm + 1e-6))      # NaN where the norm is
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    rate = m / (1.0 - beta1 ** t) / (np.sqrt(v / (1.0 - beta2 ** t)) + eps)
    return p - lr * decay * p - lr * rate, m, v


def _tops(x: np.ndarray) -> np.ndarray:
    """Each element's block's largest absolute value."""
    full = np.pad(np.abs(x.astype(np.float64)), (0, -len(x) % BLOCK)).reshape(-1, BLOCK)
    return full.max(axis=1)


def _each(tops: np.ndarray, n: int) -> np.ndarray:
    return np.repeat(tops.astype(np.float64), BLOCK)[:n]


def held_first(codes: np.ndarray, tops: np.ndarray) -> np.ndarray:
    k = codes.astype(np.float64)
    return _each(tops, len(k)) * np.sign(k) * (k / 127.0) ** 2


def held_second(codes: np.ndarray, tops: np.ndarray) -> np.ndarray:
    return _each(tops, len(codes)) * (codes.astype(np.float64) / 255.0) ** 4


def nearest_first(m: np.ndarray):
    """(codes, tops, root): root = what is rounded to the code's absolute value."""
    tops = _tops(m)
    top = _each(tops, len(m))
    root = 127.0 * np.sqrt(np.divide(np.abs(m), top, out=np.zeros_like(top), where=top > 0))
    return np.sign(m) * np.floor(root + 0.5), tops, root


def nearest_second(v: np.ndarray):
    tops = _tops(v)
    top = _each(tops, len(v))
    root = 255.0 * np.divide(v, top, out=np.zeros_like(top), where=top > 0) ** 0.25
    return np.where(v > 0, np.maximum(np.floor(root + 0.5), 1.0), 0.0), tops, root
