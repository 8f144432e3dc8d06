"""The gated delta rule in fp64, token by token from its definition (numpy; test infrastructure only).

Arrays of one (b, h): q, k [n, dk], v [n, dv], log_gate, beta [n], S [dk, dv].
"""
import numpy as np


def norm(x, axis=-1):
    return np.sqrt((x * x).sum(axis=axis))


# Sizes.  A chunked form holds S_t as a sum, of the first state and of the corrections k_i u_i^T up to t, each times the gates behind it,
# and rounds in proportion to its terms.  These may cancel (k = 1, beta = 1: the state is the last value, whatever the terms before), so what
# bounds an error is not |S_t| but the sum of the terms' norms: Z_t = a_t Z_(t-1) + |k_t| |u_t| >= |S_t|.  In the same way Y_t for the gradient
# of S_t.


def forward(q, k, v, log_gate, beta, S, scale):
    """Outputs [n, dv], the state behind the last token, the sizes of the outputs' rows and of the state."""
    S = np.array(S, dtype=np.float64)
    Z = norm(S, (0, 1))
    out, size = np.zeros((q.shape[0], v.shape[1])), np.zeros(q.shape[0])
    for t in range(q.shape[0]):
        a = np.exp(log_gate[t])
        D = a * S if a > 0 else np.zeros_like(S)
        u = beta[t] * (v[t] - D.T @ k[t])
        S = D + np.outer(k[t], u)
        Z = a * Z + norm(k[t]) * norm(u)
        out[t] = scale * (S.T @ q[t])
        size[t] = scale * norm(q[t]) * Z
    return out, S, size, Z


def backward(q, k, v, log_gate, beta, S, scale, do, dS):
    """Gradients of sum(out do) + sum(S_n dS), by name; and for each the products of norms that bound its rows."""
    n = q.shape[0]
    S = np.array(S, dtype=np.float64)
    Z = norm(S, (0, 1))
    steps = []
    for t in range(n):
        a = np.exp(log_gate[t])
        D = a * S if a > 0 else np.zeros_like(S)
        e = v[t] - D.T @ k[t]
        S = D + np.outer(k[t], beta[t] * e)
        before = a * Z
        Z = before + norm(k[t]) * norm(beta[t] * e)
        steps.append((a, D, e, S, before, Z))
    G = np.array(dS, dtype=np.float64)
    Y = norm(G, (0, 1))
    g = {"dQ": np.zeros_like(q), "dK": np.zeros_like(k), "dV": np.zeros_like(v), "dlog_gate": np.zeros(n), "dbeta": np.zeros(n)}
    size = {name: np.zeros(n) for name in g}
    for t in reversed(range(n)):
        a, D, e, S, before, Z = steps[t]
        G = G + scale * np.outer(q[t], do[t])
        Y = Y + scale * norm(q[t]) * norm(do[t])
        du = G.T @ k[t]
        u, de = beta[t] * e, beta[t] * du
        g["dQ"][t] = scale * (S @ do[t])
        g["dK"][t] = G @ u - D @ de
        g["dV"][t] = de
        g["dbeta"][t] = du @ e
        dD = G - np.outer(k[t], de)
        g["dlog_gate"][t] = (dD * D).sum()
        nk = norm(k[t])
        size["dQ"][t] = scale * Z * norm(do[t])
        size["dK"][t] = Y * norm(u) + before * norm(de)
        size["dV"][t] = abs(beta[t]) * Y * nk
        size["dbeta"][t] = Y * nk * (norm(v[t]) + before * nk)
        size["dlog_gate"][t] = (Y + nk * norm(de)) * before
        G = a * dD
        Y = a * (Y + nk * norm(de))
    g["dstate"] = G
    size["dstate"] = Y
    return g, size
