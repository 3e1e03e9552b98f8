"""The products with bit-packed weights where they could go wrong: no tokens, the widest rows, the largest activations, zero-points
beyond the codes, infinities in adapters, and how near the sums come to those in 64 bits."""
import numpy as np
import pytest
import torch

import packed_util as pu

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _tb():
    import paper_2602_04929_b200 as tb
    return tb


@pytest.mark.parametrize("dtype", [BF, F32])
def test_backward_without_tokens(dtype):
    """An empty batch has an empty dx, whether or not adapters and a kept input come with it."""
    tb = _tb()
    p = pu.problem(1, 0, 64, 96, 3, 32, dtype, 2, 8, [0, 0], [1])
    w, a = pu.on_gpu(tb, p)
    for ad in (None, a):
        dx, dA, dB = tb.tb_packed_linear_backward(w, p["dy"].cuda(), ad)
        assert dx.shape == (0, 96) and dx.dtype == dtype and dA is None and dB is None
