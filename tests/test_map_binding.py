"""What the binding of the trained map's operators does with its arguments before the library is called: no GPU."""
import numpy as np
import pytest
import torch

from paper_2212_11506_amd import _binding as b


def values(coefficients, steps):
    c = b._coefficients(coefficients, steps)
    return [c[i] for i in range(3 * steps)]


def test_coefficients_are_read_at_each_call():
    """Numbers that a caller keeps in tensors or arrays and changes in place are taken as they are now."""
    for make in (torch.tensor, lambda v: torch.tensor(v, dtype=torch.float64), np.array):
        rows = [[make(1.5), make(-0.5), make(0.0)]]
        assert values(rows, 2) == [1.5, -0.5, 0.0] * 2
        rows[0][0] += 0.25
        assert values(rows, 2) == [1.75, -0.5, 0.0] * 2
        flat = [make(1.5), make(-0.5), make(0.0)]
        assert values(flat, 1) == [1.5, -0.5, 0.0]
        flat[1] -= 0.25
        assert values(flat, 1) == [1.5, -0.75, 0.0]
    table = np.array([[2.0, -1.5, 0.5], [1.5, -0.5, 0.0]])
    assert values(table, 2) == [2.0, -1.5, 0.5, 1.5, -0.5, 0.0]
    table[1, 0] = 1.25
    assert values(table, 2) == [2.0, -1.5, 0.5, 1.25, -0.5, 0.0]
    assert values(torch.tensor([2.0, -1.5, 0.5]), 2) == [2.0, -1.5, 0.5] * 2
    assert b._coefficients(None, 5) is None


@pytest.mark.parametrize("coefficients,steps", [((1.0, 2.0), 1), ([(1.0, 2.0, 3.0)] * 2, 3), (("a", 1.0, 2.0), 1)])
def test_coefficients_are_refused(coefficients, steps):
    with pytest.raises(ValueError):
        b._coefficients(coefficients, steps)
