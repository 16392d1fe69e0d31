"""Sizes in the binding of the operators around attention that a C int cannot hold (on a host without a
GPU, with tensors that have shapes and no memory)."""
import pytest
import torch

import paper_2609_03151_amd as basp

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def _meta(*shape, dtype=F32):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32, 2 ** 32 + 64])
def test_tables_longer_than_an_int(n):
    """They come as -1, which the library refuses, and not as what is left of them in 32 bits."""
    q = _meta(1, 1, 1, 64, dtype=BF16)
    dims = basp._norm_args(q, q, None, None, _meta(n, 4), _meta(n, 4), None)[1]
    assert dims == (1, 1, 1, 1, 64, 8, -1)
    pages = _meta(3, 1, 16, 64, dtype=BF16)
    dims = basp._pages(pages, pages, None, None, _meta(2, n, dtype=I32), 2, -1)[1]
    assert dims == (1, 64, 16, 3, -1)


def test_tables_that_fit():
    q, n = _meta(1, 1, 1, 64, dtype=BF16), 2 ** 31 - 1
    assert basp._norm_args(q, q, None, None, _meta(n, 4), _meta(n, 4), None)[1][6] == n
    pages = _meta(3, 1, 16, 64, dtype=BF16)
    assert basp._pages(pages, pages, None, None, _meta(2, n, dtype=I32), 2, -1)[1][4] == n
