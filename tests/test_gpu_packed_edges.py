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


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_widest_rows(dtype):
    """2^24 columns of the result, both directions: 256 tokens of them are 2^32 values.  The last of a tile's tokens lie 255 rows from its
    first, past 2^31 values; they and others against double precision."""
    tb = _tb()
    n_tok, wide = (256, 1 << 24) if dtype == BF else (100, 1 << 24)
    g = torch.Generator(device="cuda").manual_seed(8)
    ints = lambda lo, hi, shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    looked_at = [0, n_tok // 2 - 1, n_tok // 2, n_tok - 1]

    def weights(rows, d):
        words = torch.randint(-1 << 31, 1 << 31, (rows, d // 16), generator=g, device="cuda").to(torch.int32)
        w = tb.packed_weight(words, torch.rand((rows, 1), generator=g, device="cuda") + 0.5, ints(0, 4, (rows, 1)), d, 2)
        codes = (words.unsqueeze(-1) >> torch.arange(0, 32, 2, device="cuda", dtype=torch.int32)) & 3
        return w, (codes.view(rows, d).double() - w.tensors[2]) * w.tensors[1].double()

    def check(got, v, k, weights=0.0):
        """Float sums, the result's rounding, and a rounding of every weight by `weights` of it: the last two come one after the other,
        each half a step (2^-8 in bf16) at most."""
        for t in looked_at:
            at = v[t].double()
            want, size = at @ k, at.abs() @ k.abs()
            off = (got[t].double() - want).abs()
            bound = pu.sum_bound(k.shape[0], size, dtype) + weights * size + 1.01 * pu.HALF_STEP[dtype] * (want.abs() + weights * size)
            assert (off <= bound).all(), t
            del want, size, off, bound

    # dx of 8 rows, 2 bits
    w, Q = weights(8, wide)
    dy = torch.randn((n_tok, 8), generator=g, device="cuda").to(dtype)
    dx, _, _ = tb.tb_packed_linear_backward(w, dy)
    assert tb.tb_device_error_flag() == 0
    check(dx, dy, Q, pu.HALF_STEP[BF] if dtype == BF else 0.0)
    del dx, Q, w
    # y of 2^24 rows
    w, Q = weights(wide, 32)
    x = torch.randn((n_tok, 32), generator=g, device="cuda").to(dtype)
    y, _ = tb.tb_packed_linear(w, x)
    assert tb.tb_device_error_flag() == 0
    check(y, x, Q.T)
