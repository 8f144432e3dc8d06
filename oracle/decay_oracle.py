"""Decayed linear attention and beam search in fp64, written out from their definitions (numpy; test infrastructure only).

Arrays of one (b, h): q, k [n, dk], v [n, dv], S [dk, dv]; log_decay a float.
"""
import math

import numpy as np


def power(a, n):
    """g^n for g = exp(a); g^0 = 1 also for g = 0."""
    n = np.asarray(n, dtype=np.float64)
    with np.errstate(invalid="ignore"):   # 0 * -inf
        return np.where(n == 0, 1.0, np.exp(np.where(n == 0, 0.0, a * n)))


def forward(q, k, v, a, S, scale):
    """Token by token: outputs [n, dv] and the state behind the last token."""
    g = float(power(a, 1))
    S = np.array(S, dtype=np.float64)
    out = np.zeros((q.shape[0], v.shape[1]))
    for t in range(q.shape[0]):
        S = (g * S if g > 0 else 0.0) + np.outer(k[t], v[t])
        out[t] = scale * (S.T @ q[t])
    return out, S


def weights(a, n):
    """g^(i-l) for l <= i, else 0: [n, n]."""
    apart = np.arange(n)[:, None] - np.arange(n)[None, :]
    return np.where(apart >= 0, power(a, np.maximum(apart, 0)), 0.0)


def backward(q, k, v, a, S, scale, do, dS):
    """Gradients of sum(out do) + sum(S_n dS): dq, dk, dv and that of the incoming state."""
    n = q.shape[0]
    t = np.arange(n)
    D = scale * weights(a, n)
    P, R = D * (q @ k.T), D * (do @ v.T)
    up, down = power(a, t + 1)[:, None], power(a, n - 1 - t)[:, None]
    dq = R @ k + scale * up * (do @ S.T)
    dk = R.T @ q + down * (v @ dS.T)
    dv = P.T @ do + down * (k @ dS)
    return dq, dk, dv, power(a, n) * dS + scale * (q * up).T @ do


def beam_select(logits, scores, finished=None, eos=0, keep_slots=False):
    """One batch entry: logits [n, V], scores [n]; lists (scores, parents, tokens)."""
    n, V = logits.shape
    cand = []
    for j in range(n):
        row, score = logits[j].astype(np.float64), float(scores[j])
        row = np.where(np.isnan(row), -np.inf, row)
        if not math.isfinite(score):
            score = -math.inf
        if finished is not None and finished[j]:
            value = np.full(V, -np.inf)
            value[eos] = score
        elif score == -math.inf or not np.isfinite(row.max()):
            value = np.full(V, -np.inf)
        else:
            top = row.max()
            value = score - np.log(np.exp(row - top).sum()) + (row - top)
        cand.append(value)
    cand = np.concatenate(cand)
    best = np.lexsort((np.arange(cand.size), -cand))[:n]
    picks = [(float(cand[c]), int(c // V), int(c % V)) for c in best]
    if keep_slots:
        slots, rest = [None] * n, []
        for p in picks:
            if slots[p[1]] is None:
                slots[p[1]] = p
            else:
                rest.append(p)
        picks = [p if p is not None else rest.pop(0) for p in slots]
    return [p[0] for p in picks], [p[1] for p in picks], [p[2] for p in picks]
