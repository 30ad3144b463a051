"""Sizes that 32 bits do not hold are refused by the Python calls, and not taken modulo 2^32: 2^32 + 5 rows would be turned as
five.  (Tensors without memory.)"""
import pytest
import torch

from test_paged_host import L  # noqa: F401


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32, 2 ** 32 + 5])
def test_rows(L, n):  # noqa: F811
    q = torch.empty((n, 1, 8), dtype=torch.bfloat16, device="meta")
    pos, inv = torch.empty((n,), dtype=torch.int32, device="meta"), torch.empty((4,), device="meta")
    with pytest.raises(AssertionError, match="rows"):
        L.rotary_args(q, pos, L.Rotary(inv), out=q)
    with pytest.raises(AssertionError, match="rows"):
        L.rotary(q, pos, L.Rotary(inv), out=q)


@pytest.mark.parametrize("dim", [2 ** 32 + 64, -2 ** 32 + 64, 10 ** 15, 514, 0, -2])
def test_frequencies(L, dim):  # noqa: F811
    with pytest.raises(L.LvspecError):
        L.rotary_frequencies(dim)
