"""Where top_p ends in rows whose sum lies in many small weights."""
import math

import numpy as np
import pytest
import torch

import paper_2603_04127_amd as dk
from tests.test_gpu_sample import _run

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype,V,tail,p", [
    ("bf16", 1 << 27, -25.0, 0.999),        # 2^27 weights of 2^-36: 0.19 % of the sum, of which 0.1 % of the sum is left out
    ("f32", (1 << 25) + 1, -25.6, 0.9999),  # 2^25 weights of 2^-37
    ("bf16", 1 << 20, -27.0, 0.9999995),    # 2^20 weights of 2^-39: 2^-19 of the sum
    ("f32", 131071, -22.0, 0.99999),        # 2^17 weights of 2^-32
])
def test_one_token_before_a_flat_tail(dtype, V, tail, p):
    # Equal weights are rounded alike, by 2^-33 of their value and once more by 2^-34 for their place in whole numbers.  The last token that is kept
    # has the number that top_p leaves of them: n = (p (1 + V w) - 1) / w, off by n 2^-32 < 1 for those roundings, and by 1 for the whole number.
    x = torch.full((1, V), tail, device="cuda").to(TORCH[dtype])
    x[0, 0] = 0.0
    w = math.exp(float(x[0, 1]))
    p = float(np.float32(p))
    n = 1 + math.ceil((p * (1.0 + (V - 1) * w) - 1.0) / w)
    assert 0.1 * V < n < 0.9 * V
    one = torch.ones(1, device="cuda")
    for u, want in ((1.0, n - 1), (0.0, 0)):
        token, log = dk.dark_sample(x, u * one, top_p=p, want_logprob=True)
        assert abs(int(token) - want) <= 2, (u, int(token), want)
        assert abs(float(log) - (math.log(w) if want else 0.0) + math.log(1.0 + (n - 1) * w)) <= 2.0 ** -23 * (1.0 + abs(tail))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_of_a_long_tail(dtype):
    # Weights of 1, 2^-10, 2^-20, 2^-30 by the thousandfold: each step holds about as much as the one before it, and top_p ends in each in its turn.
    parts = [(0.0, 1), (-7.0, 1000), (-14.0, 1_000_000), (-21.0, 30_000_000)]
    x = torch.cat([torch.full((n,), v) for v, n in parts]).to(TORCH[dtype])[None].cuda()
    whole = sum(n * math.exp(v) for v, n in parts)
    for p in (0.2, 0.5, 0.7, 0.95, 0.99, 0.9999):
        p = float(np.float32(p))
        left, n = p * whole, 0
        for v, count in parts:
            w = math.exp(v)
            if left <= count * w:
                n += math.ceil(left / w)
                break
            left, n = left - count * w, n + count
        # a random number of 1 draws the last that is kept; the weights' roundings, 2^-32 of their sum, in units of the one at the end
        token = int(dk.dark_sample(x, torch.ones(1, device="cuda"), top_p=p))
        assert abs(token - (n - 1)) <= 2 + 2.0 ** -32 * whole / w, (p, token, n)


@pytest.mark.parametrize("scale,temperature", [(1e38, 1e37), (1e38, 3e38), (1e38, float("inf")), (1.0, float("inf")), (1e-36, 1e-36), (1e-30, 1e-31), (1e20, 1e19), (0.0, 1.0)])
def test_sizes_of_logits_and_temperatures(scale, temperature):
    # rows drawn by the bins' way, u in the middle of a token's share (test_gpu_sample.py has the oracle's tolerance)
    rng = np.random.default_rng(3)
    x = torch.from_numpy(np.clip(scale * rng.standard_normal((4, 5001)), -3.3e38, 3.3e38).astype(np.float32))
    u = rng.random(4).astype(np.float32)
    for dtype in TORCH.values():
        for kw in (dict(top_p=0.6), dict(top_k=1500), dict(top_k=2500, top_p=0.8), dict(top_p=0.95, min_p=0.01), dict()):
            _run(x.to(dtype), u, temperature=temperature, **kw)
