"""Calls of the operators around an expert sublayer at the ends of what they allow, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import experts_reference as ref
from tests.test_experts_route import check_route

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,kept", [(4, 1), (8, 3), (8, 2), (16, 16)])
def test_groups_with_numbers_that_are_not_finite(groups, kept, scores, dtype):
    """A group whose scores are NaN comes last, but before one that is masked; +inf among the logits makes all softmax scores NaN."""
    experts, size = 64, 64 // groups
    logits = torch.randn(13, experts, generator=torch.Generator().manual_seed(8)).to(dtype)
    logits[:5, :size] = -INF  # the first group is masked
    logits[0, size * 2], logits[1, size * 2] = float("nan"), INF
    logits[2, size:] = float("nan")
    logits[3, size + 1::2] = float("nan")
    logits[4, size:size * 2] = float("nan")
    logits[5, 9], logits[6, 9] = float("nan"), INF
    logits[7, ::2] = float("nan")
    logits[8, ::3] = INF
    logits[9], logits[10] = INF, float("nan")
    logits[11, 5:40] = float("nan")
    for bias in (None, torch.linspace(-1, 1, experts).cuda()):
        for top in (1, 2):
            for renormalise in (True, False):
                e, w = check_route(logits.cuda(), min(4, kept * size), scores=scores, bias=bias, groups=groups, groups_kept=kept, group_top=top,
                                   renormalise=renormalise)
                assert (e >= 0).all(), "a masked group was kept before one with NaN"
