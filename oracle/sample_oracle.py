"""Drawing a token from a row of logits in fp64, from its definition (numpy; test infrastructure only)."""
import numpy as np


def kept(x, temperature, top_k, top_p, min_p):
    """Weights [V] of a row's logits, 0 for the tokens that are not kept."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, dtype=np.float64))
    w = np.zeros(x.size)
    live = np.nonzero(x > -np.inf)[0]
    if live.size == 0:
        return w
    order = live[np.lexsort((live, -x[live]))]   # the largest first, equal ones by their number
    top = x[order[0]]
    if not temperature > 0:
        w[order[0]] = 1.0
        return w
    with np.errstate(over="ignore", invalid="ignore"):
        e = np.where(x[order] == top, 1.0, np.exp((x[order] - top) / temperature) if np.isfinite(top) else 0.0)
    n = order.size if top_k <= 0 else min(top_k, order.size)
    e = e[:n]
    if top_p < 1:
        before = np.cumsum(e) - e
        e = e[:max(1, int((before < top_p * e.sum()).sum()))]
    if min_p > 0:
        e = np.where(e >= min(min_p, 1.0), e, 0.0)
    w[order[:e.size]] = e
    return w


def draw(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logarithm of its probability, distance of u from the nearest border between two tokens)."""
    w = kept(x, temperature, top_k, top_p, min_p)
    total = w.sum()
    if not total > 0:
        return -1, -np.inf, 1.0
    if not temperature > 0:
        return int(np.argmax(w)), 0.0, 1.0
    at = np.nonzero(w)[0]
    sums = np.cumsum(w[at]) / total
    i = min(int((sums <= max(u, 0.0)).sum()), at.size - 1)
    return int(at[i]), float(np.log(w[at[i]] / total)), float(np.abs(sums[:-1] - u).min(initial=1.0))
