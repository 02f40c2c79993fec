"""CPU oracle of the operators inside a layer, in 64 bits.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain numpy, written
from the formulas, nothing imported from the product.

  norm, norm_grad          layer norm of the rows of s, and its gradients
  bucket, bias, bias_grad  relative position bias by buckets; visible: which
                           places of the scores count
  scores, route, route_grad, balance
                           routing to experts, its gradient, the balance bias
"""
from __future__ import annotations

import math

import numpy as np


def norm(s, gamma, beta, eps):
    """(y, mean, rstd) of the rows of s."""
    s = s.astype(np.float64)
    mean = s.mean(axis=1)
    rstd = 1.0 / np.sqrt(((s - mean[:, None]) ** 2).mean(axis=1) + eps)
    return (s - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def norm_grad(dy, s, mean, rstd, gamma):
    """(dx, dgamma, dbeta), with mean and rstd as given."""
    xh = (s - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = (g - g.mean(axis=1, keepdims=True) - xh * (g * xh).mean(axis=1, keepdims=True)) * rstd[:, None]
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


# ---- relative position bias ----

def bucket(r: int, buckets: int, exact: int, distance: int, both: bool) -> int:
    n = buckets // 2 if both else buckets
    side = n if both and r > 0 else 0
    d = abs(r) if both else max(-r, 0)
    if d < exact:
        return side + d
    m = n - exact
    if m == 0:
        return side + n - 1
    # floor(m log(d / exact) / log(distance / exact)): the largest t with (d / exact)^m >= (distance / exact)^t
    t = 0
    while t < m - 1 and d ** m * exact ** (t + 1) >= exact ** m * distance ** (t + 1):
        t += 1
    return side + exact + t


def visible(batch, queries, keys, offset, causal=False, key_lengths=None, query_lengths=None):
    i, j = np.arange(queries)[:, None], np.arange(keys)[None, :]
    seen = np.ones((batch, queries, keys), dtype=bool)
    if causal:
        seen &= j <= i + offset
    for b in range(batch):
        if key_lengths is not None:
            seen[b] &= j < key_lengths[b]
        if query_lengths is not None:
            seen[b] &= i < query_lengths[b]
    return seen


def bucket_places(queries, keys, offset, *buckets):
    of = {r: bucket(r, *buckets) for r in range(-(queries - 1) - offset, keys - offset)}
    return np.array([[of[j - i - offset] for j in range(keys)] for i in range(queries)], dtype=np.int64).reshape(queries, keys)


def bias_grad(ds, seen, places, buckets):
    """(grad, magnitude), [buckets][heads]; ds: [batch][heads][queries][keys]."""
    grad = np.zeros((buckets, ds.shape[1]))
    magnitude = np.zeros_like(grad)
    for b in range(ds.shape[0]):
        for h in range(ds.shape[1]):
            x = ds[b, h][seen[b]]
            grad[:, h] += np.bincount(places[seen[b]], weights=x, minlength=buckets)
            magnitude[:, h] += np.bincount(places[seen[b]], weights=np.abs(x), minlength=buckets)
    return grad, magnitude


# ---- routing ----

SOFTMAX, SIGMOID = 0, 1


def scores(logits, score):
    x = logits.astype(np.float64)
    with np.errstate(all="ignore"):
        if score == SIGMOID:
            return 1.0 / (1.0 + np.exp(-x))
        e = np.exp(x - np.nanmax(np.where(np.isnan(x), -np.inf, x), axis=1, keepdims=True))
        e[np.isneginf(x)] = 0.0
        return e / e.sum(axis=1, keepdims=True)


def route(logits, bias, chosen, groups, kept, top, score, renormalise, scale):
    """(experts, weights): -1 and 0 in places left over."""
    T, E = logits.shape
    s = scores(logits, score)
    experts, weights = np.full((T, chosen), -1), np.zeros((T, chosen))
    for t in range(T):
        key = [float(s[t, e]) + float(bias[e]) for e in range(E)]
        free = [e for e in range(E) if not np.isneginf(logits[t, e]) and key[e] > -math.inf]
        size = E // groups
        if kept < groups:
            rank = {}
            for e in free:
                rank.setdefault(e // size, []).append(key[e])
            best = {g: sum(sorted(k, reverse=True)[:top]) for g, k in rank.items()}
            opened = sorted(best, key=lambda g: (-best[g], g))[:kept]
            free = [e for e in free if e // size in opened]
        picked = sorted(free, key=lambda e: (-key[e], e))[:chosen]
        w = np.array([s[t, e] for e in picked])
        if renormalise and len(picked):
            w = w / w.sum() if w.sum() > 0 else 0.0 * w
        experts[t, :len(picked)] = picked
        weights[t, :len(picked)] = scale * w
    return experts, weights


def route_grad(logits, experts, dweights, score, renormalise, scale):
    """(dlogits, magnitude): magnitude is the scale of rounding errors."""
    T, E = logits.shape
    s = scores(logits, score)
    out, magnitude = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        use = [n for n in range(experts.shape[1]) if 0 <= experts[t, n] < E]
        if not use:
            continue
        at = experts[t, use]
        g, w = scale * dweights[t, use], s[t, at]
        big = np.abs(g)
        if renormalise:
            total = w.sum()
            g, big = ((g - (g * w).sum() / total) / total, (big + (big * w).sum() / total) / total) if total > 0 else (0 * g, 0 * big)
        ds, dbig = np.zeros(E), np.zeros(E)
        np.add.at(ds, at, g)
        np.add.at(dbig, at, big)
        if score == SOFTMAX:
            out[t] = s[t] * (ds - (g * w).sum())
            magnitude[t] = s[t] * (dbig + (big * w).sum())
        else:
            x = logits[t].astype(np.float64)
            left = 1.0 / (1.0 + np.exp(np.minimum(x, 700.0)))
            out[t] = ds * s[t] * left
            magnitude[t] = dbig * s[t] * left
    return out, magnitude


def balance(counts, bias, rate):
    load = counts.astype(object).sum(axis=0)
    total, E = sum(load), len(load)
    step = np.array([(n * E < total) - (n * E > total) for n in map(int, load)], dtype=np.float32)
    return bias.astype(np.float32) + np.float32(rate) * step
