"""Host-side: what the binding of gated recurrence, dropout and vocabulary head refuses beside test_more_operators_abi.py."""
import pytest

from test_operators_abi import rk  # noqa: F401  (fixture)


def test_lengths_that_are_none(rk):
    """They would reach the library as 2^64 - 1, or as 0, which is one sequence."""
    import torch
    for bad in (-1, -128, 2 ** 64, 2 ** 65):
        with pytest.raises(rk.RkError):
            rk.Recur(seq_rows=bad)
    with pytest.raises(rk.RkError):
        rk.Recur(offsets=torch.zeros(3, dtype=torch.int32), seq_rows=-2)
    assert rk.Recur(seq_rows=2 ** 64 - 1)._sizes(torch.zeros(7, 8))[1] == (1, 8)
