"""Drawing tokens for as many rows as a call takes."""
import pytest
import torch

import paper_2603_04127_amd as dk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [(1 << 21) - 1, (1 << 21) + 3, 1 << 22])
def test_as_many_rows_as_a_call_takes(B):
    # 1024 threads a row: 2^32 of them for 2^22 rows, one more than a dimension of a grid holds
    g = torch.Generator(device="cuda").manual_seed(B)
    want = torch.randint(0, 3, (B,), generator=g, device="cuda")
    x = torch.full((B, 3), float("-inf"), dtype=torch.bfloat16, device="cuda").scatter_(1, want[:, None], 1.0)
    room = torch.full((B + 2,), -7, dtype=torch.int32, device="cuda")
    token = dk.dark_sample(x, torch.rand(B, generator=g, device="cuda"), out=room[1:-1])
    torch.cuda.synchronize()
    assert torch.equal(token.long(), want) and room[0] == -7 and room[-1] == -7
