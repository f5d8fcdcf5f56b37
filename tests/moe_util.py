"""A router's choice by its definition in 64 bits, token by token, apart from the library's code."""
import numpy as np


def choose(z, top, bias=None, groups=1, top_groups=1, scale=1.0, sigmoid=False, renorm=False, sum2=False):
    """z: float64 [T,E].  Returns weights float64 [T,top], experts [T,top], rows, offsets [E+1], places [T,top]."""
    T, E = z.shape
    weights, experts = np.zeros((T, top)), np.full((T, top), -1)
    for t in range(T):
        if np.isnan(z[t]).any() or (bias is not None and np.isnan(bias).any()) or (not sigmoid and np.isposinf(z[t]).any()):
            weights[t] = np.nan
            continue
        if not (z[t] > -np.inf).any():
            continue
        with np.errstate(over="ignore"):
            if sigmoid:
                s = 1.0 / (1.0 + np.exp(-z[t]))
            else:
                s = np.exp(z[t] - z[t].max())
                s = s / s.sum()
        c = z[t] if bias is None and not (groups > 1 and sum2) else s if bias is None else s + bias
        c = np.where(z[t] == -np.inf, -np.inf, c)
        if groups > 1:
            best = -np.sort(-c.reshape(groups, -1), axis=1)
            mark = best[:, 0].copy()
            if sum2 and best.shape[1] > 1:
                mark += np.where(np.isneginf(best[:, 1]), 0.0, best[:, 1])
            kept = np.argsort(-mark, kind="stable")[:top_groups]
            c = np.where(np.isin(np.arange(E) // (E // groups), kept), c, -np.inf)
        order = [e for e in np.argsort(-c, kind="stable")[:top] if c[e] > -np.inf]
        experts[t, : len(order)] = order
        w = s[order]
        weights[t, : len(order)] = w * scale / (max(w.sum(), 2.0 ** -60) if renorm else 1.0)
    flat = experts.reshape(-1)
    order = [f for f in np.argsort(flat, kind="stable") if flat[f] >= 0]
    places = np.full(T * top, -1)
    places[order] = np.arange(len(order))
    offsets = np.searchsorted(flat[order], np.arange(E + 1), side="left")
    return weights, experts, np.array(order, dtype=int) // top, offsets, places.reshape(T, top)
