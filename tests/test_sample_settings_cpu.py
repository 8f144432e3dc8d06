"""Settings of dark_sample on their way through the binding (without a GPU)."""
import pytest
import torch

import paper_2603_04127_amd as dk


@pytest.mark.parametrize("top_k,want", [(7, 7), (0, 0), (-3, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32, 2 ** 31 - 1), (2 ** 32 + 1, 2 ** 31 - 1),
                                        (10 ** 12, 2 ** 31 - 1), (-2 ** 31 - 5, 0), (-2 ** 40, 0)])
def test_top_k_beyond_32_bits_keeps_all(top_k, want):
    seen = []
    keep, dk._keep_plan = dk._keep_plan, lambda key, plan: seen.append(plan[0].top_k)
    try:
        with pytest.raises(ValueError, match="GPU"):
            dk.dark_sample(torch.zeros(2, 53), torch.zeros(2), top_k=top_k)
    finally:
        dk._keep_plan = keep
    assert seen == [want] or (want == 0 and seen[0] <= 0)
