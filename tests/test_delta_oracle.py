"""The oracle of the gated delta rule pinned by itself: recurrence = decayed linear attention where nothing is corrected, gradients = differences (CPU)."""
import numpy as np
import pytest

from oracle import decay_oracle, delta_oracle as D


def _inputs(n=9, dk=3, dv=4, seed=0):
    r = np.random.default_rng(seed)
    x = [r.standard_normal(s) for s in ((n, dk), (n, dk), (n, dv))]
    return x + [-r.random(n), r.random(n), r.standard_normal((dk, dv)), r.standard_normal((n, dv)), r.standard_normal((dk, dv))]


def test_orthogonal_keys_correct_nothing():
    # keys at right angles, an empty state: every read before a write is 0, and u_t = beta_t v_t
    n = 5
    q, _, v, _, beta, _, _, _ = _inputs(n, n, 4)
    k = np.eye(n)
    out, last, _, _ = D.forward(q, k, v, np.full(n, -0.3), beta, np.zeros((n, 4)), 0.5)
    want, state = decay_oracle.forward(q, k, beta[:, None] * v, -0.3, np.zeros((n, 4)), 0.5)
    assert np.allclose(out, want, rtol=1e-12, atol=1e-12) and np.allclose(last, state, rtol=1e-12, atol=1e-12)


def test_one_key_with_beta_one_holds_the_last_value():
    q, k, v, _, _, S, _, _ = _inputs()
    k = np.broadcast_to(k[:1] / np.linalg.norm(k[0]), k.shape)
    _, last, _, Z = D.forward(q, k, v, np.zeros(9), np.ones(9), S, 1.0)
    assert np.allclose(last.T @ k[0], v[-1], rtol=1e-12, atol=1e-12) and Z >= np.linalg.norm(last)


@pytest.mark.parametrize("gate", [None, 0.0, -np.inf])
def test_gradients_are_the_differences(gate):
    q, k, v, a, beta, S, do, dS = _inputs(seed=1)
    if gate is not None:
        a = np.full(9, gate)
    g, size = D.backward(q, k, v, a, beta, S, 0.7, do, dS)
    names = dict(q="dQ", k="dK", v="dV", a="dlog_gate", beta="dbeta", S="dstate")

    def loss(**x):
        out, last, _, _ = D.forward(*(x.get(n, y) for n, y in zip(("q", "k", "v", "a", "beta", "S"), (q, k, v, a, beta, S))), 0.7)
        return (out * do).sum() + (last * dS).sum()

    for name, x in dict(q=q, k=k, v=v, a=a, beta=beta, S=S).items():
        if name == "a" and gate == -np.inf:
            assert not g["dlog_gate"].any()
            continue
        num = np.zeros_like(x)
        for i in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[i] = 1e-5
            num[i] = (loss(**{name: x + e}) - loss(**{name: x - e})) / 2e-5
        assert np.allclose(g[names[name]], num, rtol=1e-6, atol=1e-6), name
        if name != "S":
            rows = np.abs(num) if num.ndim == 1 else np.linalg.norm(num, axis=1)
            assert (rows <= size[names[name]] * (1 + 1e-6) + 1e-6).all(), name
