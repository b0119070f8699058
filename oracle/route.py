"""Routing to experts, from its definition, in binary64: scores, the choice, the weights, the order of dispatch, and the gradient
of the weights with respect to the logits."""
from __future__ import annotations

import numpy as np

SOFTMAX, SIGMOID = 0, 1


def scores(z: np.ndarray, score: int):
    """(open experts, scores); z [T, E] binary64."""
    with np.errstate(invalid="ignore"):
        open_ = z > -np.inf
    z = np.where(open_, np.minimum(z, np.finfo(np.float32).max), -np.inf)
    if score == SIGMOID:
        with np.errstate(over="ignore"):
            return open_, np.where(open_, 1.0 / (1.0 + np.exp(-z)), 0.0)
    top = z.max(-1, keepdims=True)
    e = np.where(open_, np.exp(np.where(open_, z - np.where(np.isinf(top), 0.0, top), 0.0)), 0.0)
    return open_, e / np.maximum(e.sum(-1, keepdims=True), 1e-300)


def choose(z, k, score=SOFTMAX, bias=None, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    """ids [T, k] (-1: none), weights [T, k], and for every token the smallest distance of two keys that its choice hangs on
    (inf where equal ones are equal by their inputs)."""
    z = np.asarray(z, np.float64)
    T, E = z.shape
    open_, s = scores(z, score)
    key = np.where(open_, z if bias is None else s + np.asarray(bias, np.float64), -np.inf)
    key = np.where(key > -np.inf, key, -np.inf)                       # (a NaN bias closes too)
    by = key if group_top == 1 or bias is not None else np.where(open_, s, -np.inf)
    ids = np.full((T, k), -1, np.int64)
    gap = np.full(T, np.inf)
    size = E // groups
    for t in range(T):
        row = key[t].copy()
        if top_groups < groups:
            g = np.sort(by[t].reshape(groups, size), axis=1)[:, ::-1]
            value = g[:, 0].copy()
            if group_top == 2 and size > 1:
                value += np.where(g[:, 1] > -np.inf, g[:, 1], 0.0)
            order = np.argsort(-value, kind="stable")
            edge = value[order[top_groups - 1]] - value[order[top_groups]] if value[order[top_groups]] > -np.inf else np.inf
            if edge > 0:
                gap[t] = min(gap[t], edge)
            for x in order[top_groups:]:
                row[x * size:(x + 1) * size] = -np.inf
        order = np.argsort(-row, kind="stable")
        best = row[order[:k + 1]]
        for j in range(min(k, E)):
            if best[j] > -np.inf:
                ids[t, j] = order[j]
                if j + 1 < len(best) and best[j + 1] > -np.inf and best[j] > best[j + 1]:
                    gap[t] = min(gap[t], best[j] - best[j + 1])
    w = weights(s, ids, renorm, scale)
    return ids, w, gap


def weights(s, ids, renorm, scale):
    w = np.where(ids >= 0, np.take_along_axis(s, np.maximum(ids, 0), 1), 0.0)
    if renorm:
        w = w / np.maximum(w.sum(-1, keepdims=True), 1e-300)
    return w * scale


def dispatch(ids, E, align, rows):
    """counts, offsets, place, source of the choice `ids` [T, k]."""
    flat = ids.reshape(-1)
    counts = np.array([(flat == e).sum() for e in range(E)], np.int64)
    offsets = np.concatenate([[0], np.cumsum(-(-counts // align) * align)])
    place, source = np.full(flat.size, -1, np.int64), np.full(rows, -1, np.int64)
    for e in range(E):
        held = np.nonzero(flat == e)[0]
        place[held] = offsets[e] + np.arange(held.size)
        source[place[held]] = held
    return counts, offsets, place, source


def gradient(z, ids, dw, score=SOFTMAX, renorm=True, scale=1.0):
    """d sum(weights * dw) / dz with the choice held constant, through the Jacobians of the normalisation and of the scores."""
    z = np.asarray(z, np.float64)
    open_, s = scores(z, score)
    chosen = ids >= 0
    dw = np.where(chosen, dw, 0.0) * scale
    sel = np.where(chosen, np.take_along_axis(s, np.maximum(ids, 0), 1), 0.0)
    if renorm:
        total = np.maximum(sel.sum(-1, keepdims=True), 1e-300)
        dw = (dw - (dw * sel / total).sum(-1, keepdims=True)) / total
    ds = np.zeros_like(s)
    for t in range(z.shape[0]):
        for j in range(ids.shape[1]):
            if chosen[t, j]:
                ds[t, ids[t, j]] += dw[t, j]
    if score == SIGMOID:
        with np.errstate(over="ignore"):
            return ds * s / (1.0 + np.exp(np.where(open_, z, -np.inf)))          # 1 - s without the difference
    return s * (ds - (ds * s).sum(-1, keepdims=True))
