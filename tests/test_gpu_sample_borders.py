"""Tokens drawn by random numbers next to the borders between two tokens' shares: the oracle's, without an exception (sample_borders.py)."""
import numpy as np
import pytest
import torch

import paper_2603_04127_amd as dk
from tests import sample_borders as N

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1000, 32000, 65537, 131071])
@pytest.mark.parametrize("kw", [dict(), dict(temperature=0.7), dict(temperature=30.0), dict(top_k=400), dict(top_k=5000), dict(top_p=0.9), dict(min_p=0.01), dict(top_k=300, top_p=0.8),
                                dict(temperature=1.3, top_k=9000, top_p=0.95, min_p=0.001)])
def test_next_to_borders(kw, V, dtype):
    rng = np.random.default_rng(V)
    x = torch.from_numpy((2.5 * rng.standard_normal(V)).astype(np.float32)).to(TORCH[dtype])
    kw = {k: float(np.float32(v)) if k != "top_k" else v for k, v in kw.items()}
    u, want, log, _ = N.next_to_borders(x.double().numpy(), 128, **kw)
    assert u.size > 64
    token, got = dk.dark_sample(x.expand(u.size, V).contiguous().cuda(), torch.from_numpy(u).cuda(), want_logprob=True, **kw)
    assert (token.cpu().numpy() == want).all()
    assert (np.abs(got.double().cpu().numpy() - log) <= N.log_tolerance(log)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_next_to_borders_of_rows_with_little_in_common(dtype):
    # weights over many octaves, many equal ones, and most of a row masked
    rng = np.random.default_rng(2)
    V = 20000
    rows = [np.linspace(-30, 0, V), rng.integers(0, 40, V) / 8.0, np.where(rng.random(V) < 0.9, -np.inf, rng.standard_normal(V)), -rng.exponential(4.0, V)]
    for row in rows:
        x = torch.from_numpy(row.astype(np.float32)).to(TORCH[dtype])
        for kw in (dict(), dict(top_p=float(np.float32(0.97))), dict(top_k=1234), dict(temperature=5.0)):
            u, want, log, _ = N.next_to_borders(x.double().numpy(), 64, **kw)
            token, got = dk.dark_sample(x.expand(u.size, V).contiguous().cuda(), torch.from_numpy(u).cuda(), want_logprob=True, **kw)
            assert (token.cpu().numpy() == want).all(), kw
            assert (np.abs(got.double().cpu().numpy() - log) <= N.log_tolerance(log)).all(), kw
