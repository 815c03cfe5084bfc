"""The training operators at the edges of what they take: layouts, lengths and values at which the arithmetic of addresses,
counters and sums could go wrong, against the definitions in 64 bits where there is a result."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import train_reference as ref

BF, HF, F = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.gpu
def test_rows_that_repeat_are_refused():
    """An expanded dimension between others has distance 0, which is no distance from row to row: such a tensor (the gradient of
    a sum over tokens, say) holds fewer elements than its rows.  Dimensions of one element may have any distance."""
    x, w = torch.randn(4, 5, 16, device="cuda"), torch.ones(16, device="cuda")
    y, h, mean, rstd = rt.layer_norm(x, w)
    for wide in (torch.randn(4, 1, 16, device="cuda").expand(4, 5, 16), torch.randn(1, 5, 16, device="cuda").expand(4, 5, 16),
                 torch.randn(16, device="cuda").expand(4, 5, 16)):
        for call in (lambda: rt.dropout(wide, 0.1, 0), lambda: rt.dropout(x, 0.1, 0, out=wide), lambda: rt.layer_norm(wide, w),
                     lambda: rt.layer_norm(x, w, residual=wide), lambda: rt.layer_norm_backward(wide, h, mean, rstd, w),
                     lambda: rt.layer_norm_backward(y, wide, mean, rstd, w), lambda: rt.layer_norm_backward(y, h, mean, rstd, w, dh=wide)):
            with pytest.raises(ValueError):
                call()
    four = torch.randn(2, 3, 1, 16, device="cuda").expand(2, 3, 5, 16)
    with pytest.raises(ValueError):
        rt.dropout(four, 0.1, 0)
    one = x[:1].as_strided((1, 5, 16), (0, 16, 1))
    assert torch.equal(rt.layer_norm(one, w)[0], y[:1])
    assert torch.equal(rt.layer_norm(x[:, :1].as_strided((4, 1, 16), (80, 0, 1)), w)[0], y[:, :1])
