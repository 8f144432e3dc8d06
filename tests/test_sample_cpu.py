"""Drawing tokens: the oracle pinned by itself, and the refusals of the entry point (without a GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2603_04127_amd as dk
from oracle import sample_oracle as S

A = 1 << 20   # aligned, never dereferenced


def test_oracle_keeps_what_the_definition_says():
    x = np.log([0.1, 0.4, 0.2, 0.2, 0.1])
    assert S.kept(x, 1.0, 3, 1.0, 0.0).nonzero()[0].tolist() == [1, 2, 3]
    assert S.kept(x, 1.0, 2, 1.0, 0.0).nonzero()[0].tolist() == [1, 2]        # of equal ones the lowest token
    assert S.kept(x, 1.0, 0, 0.39, 0.0).nonzero()[0].tolist() == [1]
    assert S.kept(x, 1.0, 0, 0.41, 0.0).nonzero()[0].tolist() == [1, 2]       # the one that crosses top_p is kept
    assert S.kept(x, 1.0, 3, 0.49, 0.0).nonzero()[0].tolist() == [1]          # of the sum of those that top_k left, 0.8
    assert S.kept(x, 1.0, 0, 1.0, 0.45).nonzero()[0].tolist() == [1, 2, 3]
    assert S.kept(x, 1.0, 0, 0.0, 0.0).nonzero()[0].tolist() == [1] and S.kept(x, 0.0, 0, 1.0, 0.0).nonzero()[0].tolist() == [1]
    assert np.allclose(S.kept(x, 0.5, 0, 1.0, 0.0) * 0.16, [0.01, 0.16, 0.04, 0.04, 0.01])


def test_oracle_draws_in_the_order_of_the_tokens():
    x = np.log([0.1, 0.4, 0.2, 0.2, 0.1])
    assert [S.draw(x, u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.71, 0.89, 0.91, 1.0)] == [0, 0, 1, 1, 2, 3, 3, 4, 4]
    assert [S.draw(x, u, top_k=2)[0] for u in (0.0, 0.66, 0.67)] == [1, 1, 2]
    assert S.draw(x, 0.2, top_k=2)[1] == pytest.approx(np.log(2 / 3)) and S.draw(x, 0.7, temperature=0.0)[:2] == (1, 0.0)
    assert S.draw(np.full(3, -np.inf), 0.5)[:2] == (-1, -np.inf) and S.draw(np.array([0.0, np.inf, np.nan, np.inf]), 0.6)[0] == 3


def _p(**kw):
    base = dict(B=2, V=100, io_dtype=dk.DARK_F32, top_k=0, temperature=1.0, top_p=1.0, min_p=0.0)
    base.update(kw)
    return ctypes.byref(dk.SampleParams(*base.values()))


def test_refusals():
    f = dk.lib().dark_sample
    far = [A + (i << 20) for i in range(8)]   # logits, uniform, temperature, top_k, top_p, min_p; token, logprob
    ok = (*far, None)
    put = lambda i, x: tuple(x if j == i else y for j, y in enumerate(ok))
    nan = float("nan")
    for kw in (dict(B=-1), dict(V=0), dict(io_dtype=3), dict(temperature=-1.0), dict(temperature=nan), dict(top_p=nan), dict(min_p=nan)):
        assert f(_p(**kw), *ok) == dk.DARK_EINVAL, kw
    for kw in (dict(V=(1 << 27) + 1), dict(B=(1 << 22) + 1)):
        assert f(_p(**kw), *ok) == dk.DARK_EUNSUPPORTED, kw
    assert f(None, *ok) == dk.DARK_EINVAL
    for i in (0, 1, 6):
        assert f(_p(), *put(i, None)) == dk.DARK_EINVAL, i
    assert f(_p(), far[0], None, None, *far[3:], None) == dk.DARK_EINVAL            # no random numbers, a temperature above 0
    assert f(_p(temperature=0.0), far[0], None, *far[2:], None) == dk.DARK_EINVAL   # an array may say otherwise
    for i in range(8):
        assert f(_p(), *put(i, far[i] + 2)) == dk.DARK_EALIGN, i
    assert f(_p(), *put(0, far[0] + 8)) == dk.DARK_EALIGN
    for result in (6, 7):
        for other in range(result):
            assert f(_p(), *put(result, far[other])) == dk.DARK_EINVAL, (result, other)
    assert f(_p(), *put(6, far[0] + 2 * 100 * 4 - 4)) == dk.DARK_EINVAL   # in the last row's last logit
    assert f(_p(B=0), *(None,) * 9) == dk.DARK_OK


def test_binding_refusals():
    x, u = torch.zeros(2, 50), torch.zeros(2)
    with pytest.raises(ValueError, match="uniform"):
        dk.dark_sample(x, u.double())
    with pytest.raises(ValueError, match="temperature"):
        dk.dark_sample(x, u, temperature=torch.zeros(3))
    with pytest.raises(ValueError, match="top_k"):
        dk.dark_sample(x, u, top_k=torch.zeros(2))
    with pytest.raises(ValueError, match="out"):
        dk.dark_sample(x, u, out=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError):
        dk.dark_sample(x.half(), u)
    with pytest.raises(ValueError, match="GPU"):
        dk.dark_sample(x, u)
    with pytest.raises(ValueError):
        dk.dark_sample(x[0], u)
