"""Which kernel a product with bit-packed weights goes to, as the scratch that it asks for shows: tiles need some, the kernel for few tokens
none (a query of shapes: runs without a GPU)."""
import ctypes

import pytest

import paper_2602_04929_b200 as tb


def tiles(n_tok, rows, d, rank=0, bits=4):
    w = tb.PackedWeight(rows, d, bits, 128, None, None, None)
    a = tb.Adapters(4, rank, n_tok, None, None, None, None, None) if rank else None
    return tb.load().tb_packed_linear_workspace(ctypes.addressof(w), ctypes.addressof(a) if rank else None, 1, n_tok) > 0


@pytest.mark.parametrize("rows,d", [(4096, 4096), (8192, 8192), (8192, 512), (512, 8192), (1024, 1024)])
def test_few_tokens_without_adapters(rows, d):
    assert not any(tiles(n, rows, d) for n in range(1, 33))


@pytest.mark.parametrize("rows,d", [(4096, 4096), (8192, 8192), (8192, 512), (512, 8192), (1024, 1024)])
@pytest.mark.parametrize("rank", [8, 64, 128])
def test_eight_tokens_of_any_rank(rows, d, rank):
    assert not any(tiles(n, rows, d, rank) for n in range(1, 9))


def test_more_tokens_by_tokens_x_columns_x_rank():
    """The measured side of either, where they differ by more than a few per cent."""
    for few in ((16, 4096, 4096, 16), (16, 4096, 4096, 64), (32, 8192, 512, 16), (32, 1024, 1024, 128), (256, 1024, 1024, 16)):
        assert not tiles(*few), few
    for many in ((24, 4096, 4096, 128), (32, 4096, 4096, 128), (32, 4096, 4096, 64), (24, 8192, 8192, 64), (32, 8192, 8192, 128), (32, 8192, 512, 64),
                 (32, 8192, 512, 128), (64, 4096, 4096, 16)):
        assert tiles(*many), many
