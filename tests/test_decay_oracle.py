"""The oracle of decayed linear attention pinned by itself: recurrence = weights written out, gradients = differences (CPU)."""
import numpy as np
import pytest

from oracle import decay_oracle as D


def _inputs(n=9, dk=3, dv=4, seed=0):
    r = np.random.default_rng(seed)
    return [r.standard_normal(s) for s in ((n, dk), (n, dk), (n, dv), (dk, dv), (n, dv), (dk, dv))]


@pytest.mark.parametrize("a", [0.0, -0.3, -40.0, -np.inf])
def test_recurrence_is_the_weighted_sum(a):
    q, k, v, S, _, _ = _inputs()
    out, last = D.forward(q, k, v, a, S, 0.5)
    t = np.arange(9)
    want = 0.5 * (D.weights(a, 9) * (q @ k.T)) @ v + 0.5 * D.power(a, t + 1)[:, None] * (q @ S)
    assert np.allclose(out, want, rtol=1e-12, atol=1e-12)
    assert np.allclose(last, D.power(a, 9) * S + (k * D.power(a, 8 - t)[:, None]).T @ v, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("a", [0.0, -0.3, -np.inf])
def test_gradients_are_the_differences(a):
    q, k, v, S, do, dS = _inputs(seed=1)
    grads = dict(zip("qkvS", D.backward(q, k, v, a, S, 0.7, do, dS)))

    def loss(**x):
        out, last = D.forward(x.get("q", q), x.get("k", k), x.get("v", v), a, x.get("S", S), 0.7)
        return (out * do).sum() + (last * dS).sum()

    for name, x in dict(q=q, k=k, v=v, S=S).items():
        num = np.zeros_like(x)
        for i in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[i] = 1e-3   # the loss is linear in each of them
            num[i] = (loss(**{name: x + e}) - loss(**{name: x - e})) / 2e-3
        assert np.allclose(grads[name], num, rtol=1e-9, atol=1e-9), name


def test_beam_ties_go_to_the_lowest_index():
    logits = np.zeros((2, 5))
    assert D.beam_select(logits, [-1.0, -1.0])[1:] == ([0, 0], [0, 1])
    assert D.beam_select(logits, [-2.0, -1.0], keep_slots=True)[1:] == ([1, 1], [1, 0])
    s, p, t = D.beam_select(logits, [-1.0, -np.inf], finished=[1, 0], eos=3)
    assert (s, p, t) == ([-1.0, -np.inf], [0, 0], [3, 0])
