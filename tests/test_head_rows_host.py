"""Rows of heads whose number is one: the distance to the next is nobody's (host tensors; nothing runs)."""
import pytest
import torch

from paper_2609_33503_b200 import binding as B
from tests.test_continuations_binding import bf


def test_one_row_of_fused_rows_is_laid_out_like_one_by_itself():
    """Queries, keys and values of one token, cut from a fused projection, beside outputs of their own."""
    fused = bf(5, 12, 64)
    q, own = fused[2:3, :8], bf(1, 8, 64)
    assert q.stride() != own.stride()
    for x, like in ((q, own), (own, q), (q, q), (q, None)):
        n, heads, dim, token, head = B._head_rows(x, like, 1, 8, 64)
        assert (n, heads, dim, head) == (1, 8, 64, 64) and token >= 64 and token % 8 == 0
    with pytest.raises(ValueError, match="laid out"):
        B._head_rows(fused[2:4, :8], bf(2, 8, 64), None, None, None)


def test_one_head_of_many_is_laid_out_like_one_by_itself():
    many = bf(6, 3, 128)
    x, own = many[:, 1:2], torch.as_strided(bf(6 * 3 * 128), (6, 1, 128), (384, 128, 1))
    odd = torch.as_strided(bf(6 * 3 * 128), (6, 1, 128), (384, 131, 1))          # (a distance that no heads could have)
    for a, b in ((x, own), (own, x), (x, odd), (odd, x)):
        n, heads, dim, token, head = B._head_rows(a, b, 6, 1, 128)
        assert (n, heads, dim, token) == (6, 1, 128, 384) and head >= 128 and head % 8 == 0
    with pytest.raises(ValueError, match="laid out"):
        B._head_rows(x, bf(6, 1, 128), None, None, None)                         # (rows 384 apart, and 128)


def test_one_row_whose_distance_no_rows_could_have():
    x = torch.as_strided(bf(400), (1, 2, 64), (131, 64, 1))
    assert B._head_rows(x, None, None, None, None) == (1, 2, 64, 64, 64)


def test_no_rows_are_laid_out_like_any():
    assert B._head_rows(bf(5, 12, 64)[2:2, :8], bf(0, 8, 64), 0, 8, 64)[:3] == (0, 8, 64)
