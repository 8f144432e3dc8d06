"""Close bounds for the gated delta rule: errors against the terms that the chunks' sums have, in the root mean square.

A chunk takes a state S, held to 24 bits, and adds k_i u_i^T to it; what a result of its token t is read from is S_t, a sum of these terms whose roundings are of
either sign: a share r of the root of the sum of their squares.  Where the terms cancel (one key and beta 2: u_t turns its sign from token to token), this is more than a share r of what they
leave, and so the error that a chunk leaves in its last state.  A later token takes that error times a (I - beta k k^T), which shortens it (beta |k|^2 <= 2) or,
at right angles to k, leaves it as it is, times the gate.  Errors of different chunks have nothing to do with each other: their squares add up.  So the error of S_t is r z_t at most,
  z_t^2 = (sum over the chunks up to t) (gates behind the chunk's start)^2 |S|^2 + (sum over i <= t) (gates behind i)^2 |k_i|^2 |u_i|^2,
spread over its dk dv elements, and that of the gradient G_t of S_t r y_t, made up alike from the other end.  Read along a direction that has nothing to do with
the error, sums over dk elements give 1 / sqrt(dk) of it:
  out_t      scale |q| z / sqrt(dk)               dQ_t   scale |dO| z / sqrt(dv)            dV_t   |beta| |k| y / sqrt(dk)
  dK_t       (|u| y + |de| z_(t-1) a) / sqrt(dv), de = beta G^T k
  dbeta_t    its two factors du = G^T k and e = v - a S_(t-1)^T k, each with the other's error: |e| |k| y / sqrt(dk dv) and |du| (|v|^2 / dv + (|k| a z_(t-1))^2 / (dk dv))^(1/2)
  dgate_t    |dD| |D| / sqrt(dk dv) of D = a S_(t-1) and its gradient dD = G - k de^T, by z and y
With keys that are all alike the errors lie along them: then `aligned`, without the 1 / sqrt(dk) where keys read.

r: four products one after the other (K S, T R, K^T U, the inverse T), each with sums of up to 320 terms.  The roundings of a sum of n terms of either sign, 2^-24 / sqrt(3)
of sums that grow with the root of their number, are sqrt(n / 2) 2^-24 / sqrt(3) of it together: 2^-21.1, 2^-20.1 for four; planes add 2^-23 each, exponentials 2^-22. A factor
of four beside 2^-20 for shares that are not even: r = 2^-18.  A result takes it twice at most (two factors): 2 r for all of a tensor, and for the worst row or number, of up to 10^5 of
a bell curve, four times that.
bf16 results: their rounding, 2^-8 / sqrt(3) of the value in the root mean square and 2^-8 at most (half a step is 2^-9 to 2^-8 of it), and 16 bits of what goes into them alone: 2^-15 of the terms
for two operands of two truncated planes.
"""
import numpy as np

from oracle.delta_oracle import norm
from tests import delta_util as U

R = 2.0 ** -18
CHUNK = {"f32": 32, "bf16": 64}


def sizes(q, k, v, log_gate, beta, S, scale, do, dS, C, aligned):
    """For one (b, h) the root mean square of the terms of every result's rows."""
    n, dk = q.shape
    dv = v.shape[1]
    rk, rv = 1.0 if aligned else dk ** -0.5, dv ** -0.5
    a = np.exp(log_gate)
    S, G = np.array(S, dtype=np.float64), np.array(dS, dtype=np.float64)
    z2, steps = 0.0, []
    for t in range(n):
        if t % C == 0:
            z2 += (S * S).sum()
        D = a[t] * S if a[t] > 0 else np.zeros_like(S)
        e = v[t] - D.T @ k[t]
        S = D + np.outer(k[t], beta[t] * e)
        before = a[t] ** 2 * z2
        z2 = before + (norm(k[t]) * norm(beta[t] * e)) ** 2
        steps.append((e, np.sqrt(before), np.sqrt(z2)))
    size = {name: np.zeros(n) for name in U.ROWS}
    size["last"] = np.sqrt(z2 + (S * S).sum())
    y2 = 0.0
    for t in reversed(range(n)):
        if t % C == C - 1 or t == n - 1:
            y2 += (G * G).sum()
        e, before, z = steps[t]
        G = G + scale * np.outer(q[t], do[t])
        y2 = y2 + (scale * norm(q[t]) * norm(do[t])) ** 2
        y, nk = np.sqrt(y2), norm(k[t])
        du = G.T @ k[t]
        de = beta[t] * du
        size["out"][t] = scale * norm(q[t]) * z * rk
        size["dQ"][t] = scale * norm(do[t]) * z * rv
        size["dV"][t] = abs(beta[t]) * nk * y * rk
        size["dK"][t] = (norm(beta[t] * e) * y + norm(de) * before) * rv
        size["dbeta"][t] = np.sqrt((norm(e) * nk * y * rk * rv) ** 2 + norm(du) ** 2 * ((norm(v[t]) * rv) ** 2 + (nk * before * rk * rv) ** 2))
        y2 = y2 + (nk * norm(de)) ** 2
        size["dlog_gate"][t] = np.sqrt(y2) * before * rv * (1.0 if aligned else dk ** -0.5)
        G = a[t] * (G - np.outer(k[t], de)) if a[t] > 0 else np.zeros_like(G)
        y2 = a[t] ** 2 * y2
    size["dstate"] = np.sqrt(y2 + (G * G).sum())
    return size


def sizes_of(p, scale=0.0, aligned=False):
    Q, K, V, dO, a, beta = (U.f64(p[x]) for x in U_NAMES)
    B, H, L, dk = Q.shape
    dv, scale = V.shape[3], scale or dk ** -0.5
    r = {x: np.zeros((B, H, L)) for x in U.ROWS}
    r["last"], r["dstate"] = np.zeros((B, H)), np.zeros((B, H))
    S, dS = (np.zeros((B, H, dk, dv)) if p[x] is None else U.f64(p[x]) for x in ("state", "dstate"))
    for b in range(B):
        n = L if p["lengths"] is None else min(max(int(p["lengths"][b]), 0), L)
        for h in range(H):
            one = sizes(*(x[b, h, :n] for x in (Q, K, V, a, beta)), S[b, h], scale, dO[b, h, :n], dS[b, h], CHUNK[p["dtype"]], aligned or dk == 1)
            for x, t in one.items():
                if x in ("last", "dstate"):
                    r[x][b, h] = t
                else:
                    r[x][b, h, :n] = t
    return r


U_NAMES = ("Q", "K", "V", "dOut", "a", "beta")


def excess(got, want, size, dtype, what):
    """Errors in units of what is allowed: of the whole tensor, and of its worst row."""
    g = np.asarray(got, dtype=np.float64) if isinstance(got, np.ndarray) else U.f64(got)
    assert g.shape == want.shape and np.isfinite(g).all(), what
    axes = () if what in ("dlog_gate", "dbeta") else (-1, -2) if what in ("last", "dstate") else (-1,)
    rows = lambda x: np.abs(x) if not axes else np.sqrt((x * x).sum(axes))
    err, ref = rows(g - want), rows(want)
    narrow = dtype == "bf16" and what in ("out", "dQ", "dK", "dV")
    share = 2 * R + (2.0 ** -15 if narrow else 0.0)
    whole = share * np.sqrt((size ** 2).sum()) + (2.0 ** -8 / np.sqrt(3) * 1.05 * np.sqrt((ref ** 2).sum()) if narrow else 0.0)
    worst = 4 * share * size + (2.0 ** -8 * ref if narrow else 0.0)
    tiny = 1e-37 * np.sqrt(max(1, want.size))   # results below the smallest normal numbers
    return float(np.sqrt((err ** 2).sum()) / (whole + tiny)) if want.size else 0.0, float((err / (worst + tiny)).max(initial=0.0))


def check(got, want, size, dtype, what):
    whole, worst = excess(got, want, size, dtype, what)
    print(f"{what}: {whole:.3f} of what is allowed, worst row {worst:.3f}")
    assert whole <= 1.0 and worst <= 1.0, (what, whole, worst)
