"""The comparisons of tests/helpers.py fail on what is no number (no GPU needed)."""
import numpy as np
import pytest
import torch

from helpers import rel_fro_of_numbers, within

NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("bad", [NAN, INF, -INF, 2.0])
def test_within(bad):
    want, err = torch.tensor([1.0, -3.0, 0.0], dtype=torch.float64), torch.tensor([0.0, 1e-3, 1e-3], dtype=torch.float64)
    within(torch.tensor([1.0 + 2.0 ** -9, -3.0005, 1e-4]), want, err, 2.0 ** -8)
    for i in range(3):
        got = want.clone()
        got[i] = bad
        with pytest.raises(AssertionError):
            within(got, want, err, 2.0 ** -8)
    with pytest.raises(AssertionError):
        within(torch.full((3,), bad), want, err, 2.0 ** -8)


@pytest.mark.parametrize("bad", [NAN, INF])
def test_rel_fro_of_numbers(bad):
    want = np.array([[1.0, 2.0], [3.0, 4.0]])
    assert rel_fro_of_numbers(want, want) == 0.0
    for a, b in ((np.array([[1.0, 2.0], [bad, 4.0]]), want), (want, np.full((2, 2), bad))):
        with pytest.raises(AssertionError):
            rel_fro_of_numbers(a, b)
