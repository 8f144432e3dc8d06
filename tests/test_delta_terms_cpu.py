"""The close bounds of the gated delta rule's results: the chunked formulas in fp64 give the oracle's results, and results with a term left out, rows of zeros or
noise do not pass the bounds (CPU)."""
import numpy as np
import pytest

from tests import delta_terms as T, delta_util as U

NAMES = ("dQ", "dK", "dV", "dlog_gate", "dbeta")


def _chunked(q, k, v, log_gate, beta, S, scale, do, dS, C, without=()):
    """Gradients of one (b, h) by the chunked formulas; `without`: names of terms that are left out of the gradients of gates and betas, of dK and dQ."""
    n = q.shape[0]
    states, parts = [], []
    for c0 in range(0, n, C):
        x = slice(c0, min(c0 + C, n))
        K, Q, V, b = k[x], q[x], v[x], beta[x]
        m = K.shape[0]
        G = np.cumsum(log_gate[x])
        D = np.tril(np.exp(G[:, None] - G[None]))
        E = np.tril(D * (K @ K.T), -1)
        Ti = np.linalg.inv(np.eye(m) + b[:, None] * E)
        P, gamma, left = D * (Q @ K.T), np.exp(G), np.exp(G[-1] - G)
        u = Ti @ (b[:, None] * (V - gamma[:, None] * (K @ S)))
        states.append(S)
        parts.append((x, K, Q, V, b, D, E, Ti, P, gamma, left, u))
        S = np.exp(G[-1]) * S + K.T @ (left[:, None] * u)
    g = {"dQ": np.zeros_like(q), "dK": np.zeros_like(k), "dV": np.zeros_like(v), "dlog_gate": np.zeros(n), "dbeta": np.zeros(n)}
    for (x, K, Q, V, b, D, E, Ti, P, gamma, left, u), S in zip(reversed(parts), reversed(states)):
        dO, m, Gamma = do[x], K.shape[0], gamma[-1]
        dR = Ti.T @ (scale * P.T @ dO + left[:, None] * (K @ dS))
        N = scale * D * (dO @ u.T)
        M = -b[:, None] * np.tril(D * (dR @ u.T), -1)
        X1, X2, X3 = scale * gamma[:, None] * (dO @ S.T), gamma[:, None] * (dR @ S.T), left[:, None] * (u @ dS.T)
        g["dQ"][x] = X1 + (0 if "N K" in without else N @ K)
        g["dK"][x] = X3 - b[:, None] * X2 + (0 if "M K" in without else M @ K) + (0 if "MT K" in without else M.T @ K) + (0 if "NT Q" in without else N.T @ Q)
        g["dV"][x] = b[:, None] * dR
        F = np.tril(D * (dR @ u.T), -1)
        g["dbeta"][x] = (dR * V).sum(1) - (0 if "S dR" in without else (K * X2).sum(1)) - (0 if "E dR.u" in without else ((K @ K.T) * F).sum(1))
        Z = np.tril((Q @ K.T) * N, -1) - b[:, None] * (K @ K.T) * F      # weight (r, i) times its gradient
        reads = (Q * X1).sum(1) - b * (K * X2).sum(1)
        kept = (K * X3).sum(1)
        for t in range(m):
            gate = 0.0
            if "pairs" not in without:
                gate += Z[t:, :t].sum()
            if "reads" not in without:
                gate += reads[t:].sum()
            if "kept" not in without:
                gate += kept[:t].sum()
            if "S dS" not in without:
                gate += Gamma * (S * dS).sum()
            g["dlog_gate"][x.start + t] = gate
        dS = Gamma * dS + scale * Q.T @ (gamma[:, None] * dO) - K.T @ ((gamma * b)[:, None] * dR)
    return g


def _case(dtype, L, wide, **kw):
    p = U.problem(L + wide, 1, 1, L, wide, wide, dtype, state=True, dstate=True, **kw)
    x = [U.f64(p[k])[0, 0] for k in ("Q", "K", "V", "a", "beta")]
    rest = (U.f64(p["state"])[0, 0], wide ** -0.5, U.f64(p["dOut"])[0, 0], U.f64(p["dstate"])[0, 0], T.CHUNK[dtype])
    want, _ = U.oracle(p)
    return p, (*x, *rest), {k: want[k] for k in NAMES}


CASES = [("f32", 65, 64, {}), ("f32", 200, 32, {}), ("f32", 515, 64, {}), ("bf16", 65, 64, {}), ("bf16", 200, 128, {}), ("bf16", 515, 64, {}),
         ("f32", 170, 64, dict(beta=2.0, same_key=True, keys=0.99)), ("bf16", 170, 64, dict(beta=2.0, same_key=True, keys=0.99)), ("bf16", 170, 64, dict(beta=1.0, same_key=True))]


@pytest.mark.parametrize("dtype,L,wide,kw", CASES)
def test_what_passes_and_what_does_not(dtype, L, wide, kw):
    p, args, want = _case(dtype, L, wide, **kw)
    size = T.sizes_of(p, aligned=bool(kw))

    def passes(name, got):
        return max(T.excess(got[None, None], want[name], size[name], dtype, name)) <= 1.0

    g = _chunked(*args)
    for name in NAMES:
        assert np.allclose(g[name], want[name][0, 0], rtol=1e-8, atol=1e-8 * np.abs(want[name]).max()), name
        assert passes(name, g[name]), name
    for term, name in (("pairs", "dlog_gate"), ("reads", "dlog_gate"), ("kept", "dlog_gate"), ("S dS", "dlog_gate"), ("S dR", "dbeta"), ("E dR.u", "dbeta"), ("M K", "dK"),
                       ("MT K", "dK"), ("NT Q", "dK"), ("N K", "dQ")):
        assert not passes(name, _chunked(*args, without=(term,))[name]), term
    rng = np.random.default_rng(0)
    for name in NAMES:
        zeros = want[name][0, 0].copy()
        zeros[rng.random(L) < 0.1] = 0.0
        assert not passes(name, zeros), name
        one = want[name][0, 0].copy()
        one[L // 2] = 0.0   # a single row
        assert not passes(name, one), name
        if dtype == "f32" or name in ("dlog_gate", "dbeta"):
            assert not passes(name, want[name][0, 0] * (1.0 + 2.0 ** -9 * rng.standard_normal(want[name][0, 0].shape))), name
