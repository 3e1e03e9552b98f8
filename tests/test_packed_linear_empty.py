"""An empty batch through the products with bit-packed weights: nothing to do and no error (found on the host: runs without a GPU)."""
import ctypes

import paper_2602_04929_b200 as tb

ONE = 256
W = tb.PackedWeight(256, 512, 4, 128, ONE, ONE, ONE)
A = tb.Adapters(3, 16, 2, ONE, ONE, ONE, ONE, ONE)


def backward(a=None, n=0, dx=None, dA=None, dB=None):
    """Arrays of tokens are NULL, as empty tensors are."""
    return tb.load().tb_packed_linear_backward(ctypes.addressof(W), a, None, 1, n, None, None, None, None, dx, dA, dB, None, 0, None)


def test_backward_of_no_tokens():
    assert backward() == 0
    assert backward(ctypes.addressof(A)) == 0
    assert backward(dA=ONE, dB=ONE) == 1                        # gradients of adapters without adapters
    assert backward(ctypes.addressof(A), dA=ONE) == 1           # dA and dB come together


def test_a_backward_call_that_asks_for_nothing_is_refused():
    assert backward(n=5) == 1
    assert backward(ctypes.addressof(A), n=5) == 1
