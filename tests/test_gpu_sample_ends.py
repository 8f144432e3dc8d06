"""Random numbers at the ends of 0 ... 1: the first and the last token that is kept, however little they weigh."""
import numpy as np
import pytest
import torch

import paper_2603_04127_amd as dk
from oracle import sample_oracle as S

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(), dict(top_k=300), dict(top_k=4000), dict(min_p=1e-30), dict(temperature=0.9, top_k=500, min_p=1e-35)])
def test_the_first_and_the_last_token_that_is_kept(kw, dtype):
    # The tokens at both ends weigh 2^-60 to 2^-86 of the others: the sums before the last are those of all to 64 bits, give or take a rounding.
    rng = np.random.default_rng(5)
    V = 5000
    x = rng.standard_normal((64, V)).astype(np.float32)
    x[:, :600] -= 50.0
    x[:, 4400:] -= 50.0
    if "top_k" in kw:   # few others, so that the ends are among those that are kept
        x[:, kw["top_k"] // 2:4300] = -np.inf
    x = torch.from_numpy(x).to(TORCH[dtype])
    first, last = [], []
    for row in x.double().numpy():
        kept = np.nonzero(S.kept(row, **{**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **{k: float(np.float32(v)) if k != "top_k" else v for k, v in kw.items()}}))[0]
        first.append(kept[0])
        last.append(kept[-1])
    x = x.cuda()
    ones = torch.ones(64, device="cuda")
    for u, want in ((1.0, last), (2.0, last), (0.0, first), (-1.0, first)):
        token = dk.dark_sample(x, u * ones, **kw).cpu().numpy()
        assert (token == np.array(want)).all(), (u, token, want)
