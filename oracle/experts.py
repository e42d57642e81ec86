"""A feed-forward block made of experts in plain fp64 numpy (TEST INFRASTRUCTURE ONLY, as oracle/ops.py): the choice of
experts, the grouping of the chosen pairs, the products slot by slot, the weighted sum.
"""
from __future__ import annotations

import numpy as np

from oracle import ops


def scores(l, sigmoid):
    """One row's scores; 0 where the logit rules out."""
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    l = np.minimum(l, float(np.finfo(np.float32).max))
    s = np.zeros(len(l))
    live = l > -np.inf
    if sigmoid:
        s[live] = 1 / (1 + np.exp(-np.maximum(l[live], -80)))
    elif live.any():
        with np.errstate(over="ignore"):
            s[live] = np.exp(l[live] - l[live].max())
        s /= s.sum()
    return s


def choose(l, top_k, sigmoid=False, bias=None, groups=1, top_groups=1, renorm=True, scale=1.0):
    """(experts, weights) of one row, -1 and 0 where none is left."""
    n = len(l)
    s = scores(l, sigmoid)
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    v = s if bias is None else s + bias
    live = [e for e in range(n) if l[e] > -np.inf and v[e] > -np.inf]
    if top_groups < groups:
        each = n // groups
        sums = []
        for g in range(groups):
            best = sorted((v[e] for e in live if e // each == g), reverse=True)[:2]
            sums.append((-sum(best), g) if best else (np.inf, g))
        keep = {g for _, g in sorted(sums)[:top_groups]}
        live = [e for e in live if e // each in keep]
    # (a sigmoid takes a logit as -80 at least, +inf is the largest finite number)
    by = np.minimum(np.maximum(l, -80) if sigmoid else l, float(np.finfo(np.float32).max)) if bias is None else v
    chosen = sorted(live, key=lambda e: (-by[e], e))[:top_k]
    expert, weight = np.full(top_k, -1, np.int64), np.zeros(top_k)
    expert[:len(chosen)] = chosen
    w = s[chosen]
    if renorm and len(chosen):
        if not sigmoid:     # (the chosen may all be far below the largest logit)
            x = np.minimum(l[chosen], float(np.finfo(np.float32).max))
            w = np.exp(x - x.max())
        w = w / w.sum()
    weight[:len(chosen)] = scale * w
    return expert, weight


def group(expert, experts):
    """(offsets, order, place) of chosen experts [rows][top_k]."""
    flat = expert.reshape(-1)
    order = [p for e in range(experts) for p in np.flatnonzero(flat == e)]
    offsets = np.concatenate([[0], np.cumsum([(flat == e).sum() for e in range(experts)])])
    place = np.full(len(flat), -1)
    place[order] = np.arange(len(order))
    return offsets, np.array(order + [-1] * (len(flat) - len(order))), place.reshape(expert.shape)


def expert_of(offsets):
    """Each slot's expert."""
    return np.repeat(np.arange(len(offsets) - 1), np.diff(offsets))


def combine(y, weight, place, add=None):
    """out[t] = add[t] + sum_j weight[t][j] y[place[t][j]]."""
    out = np.zeros((len(place), y.shape[1])) if add is None else add.copy()
    for t, at in enumerate(place):
        for j, p in enumerate(at):
            if 0 <= p < len(y):
                out[t] += weight[t, j] * y[p]
    return out


def block(x, l, w_gate, w_up, w_down, **settings):
    """The whole block for rows x [T][H] and logits l: the sum of the chosen experts' results (no 8-bit roundings
    between the products)."""
    out = np.zeros((len(x), len(w_down[0])))
    for t in range(len(x)):
        for e, w in zip(*choose(l[t], **settings)):
            if e >= 0:
                out[t] += w * (ops.gated(x[t:t + 1], w_gate[e], w_up[e])[2] @ w_down[e].T)[0]
    return out
