"""What the numbers next to the borders tell apart (CPU): sums of 32 bits, or weights of one half off by 2^-25, draw other tokens than the definition."""
import numpy as np
import pytest

from oracle import sample_oracle as S
from tests import sample_borders as N


def _draw(w, u):
    at = np.nonzero(w)[0]
    sums = np.cumsum(w[at]) / w[at].sum()
    i = np.minimum(np.searchsorted(sums, u.astype(np.float64), side="right"), at.size - 1)
    return at[i], np.log(w[at[i]] / w[at].sum())


@pytest.mark.parametrize("kw", [dict(), dict(temperature=0.7), dict(top_k=5000), dict(top_p=0.9), dict(min_p=0.01)])
def test_weights_that_are_a_little_off(kw):
    rng = np.random.default_rng(1)
    x = (2.5 * rng.standard_normal(40000)).astype(np.float32).astype(np.float64)
    u, token, log, gap = N.next_to_borders(x, 256, **kw)
    assert u.size == 256 and (gap > N.NEAR).all() and np.median(gap) < 2.0 ** -26
    w = S.kept(x, **{**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **kw})
    assert (_draw(w, u)[0] == token).all()
    assert all(S.draw(x, float(a), **kw)[0] == t for a, t in zip(u[:8], token))
    assert (_draw(w * (1.0 + 2.0 ** -32 * rng.uniform(-1, 1, w.size)), u)[0] == token).all()          # as good as the library says its weights are
    other = w * (1.0 + 2.0 ** -25 * (np.arange(w.size) < w.size // 2))   # one half of the row off by 2^-25
    assert (_draw(other, u)[0] != token).any()
    at = np.nonzero(w)[0]
    single = np.cumsum((w[at] / w[at].sum()).astype(np.float32), dtype=np.float32).astype(np.float64)   # sums of 32 bits
    assert (at[np.minimum(np.searchsorted(single / single[-1], u.astype(np.float64), side="right"), at.size - 1)] != token).any()
    assert not (2.0 ** -18 <= N.log_tolerance(log)).any()
