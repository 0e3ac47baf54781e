"""The float64 reference of the distillation loss against values worked out by
hand where its terms leave float64's range (no GPU)."""
import numpy as np
import pytest

from oracle import sequence as S


@pytest.mark.parametrize("shift", [0.0, -100.0, -800.0, -5000.0])
def test_a_list_that_is_made_to_sum_to_1_has_its_proportions_at_any_level(shift):
    """q depends on differences of the listed logps only."""
    x = np.array([[0.3, -1.0, 2.0, 0.0]])
    idx = np.array([[2, 0]])
    lp = np.array([[0.0, np.log(0.25)]])
    loss, grad = S.distill_top(x, lp + shift, idx)
    p = np.exp(x[0]) / np.exp(x[0]).sum()
    want = 0.8 * np.log(0.8 / p[2]) + 0.2 * np.log(0.2 / p[0])
    assert abs(loss[0] - want) < 1e-12
    assert np.abs(grad[0] - (p - [0.2, 0.0, 0.8, 0.0])).max() < 1e-12


def test_a_list_of_probability_0_teaches_nothing():
    x = np.array([[0.3, -1.0, 2.0, 0.0]])
    for tail in (False, True):
        for idx, lp in (([[0, 1]], [[-np.inf, -np.inf]]), ([[-1, 4]], [[0.0, 0.0]])):
            loss, grad = S.distill_top(x, np.array(lp), np.array(idx), tail=tail)
            assert loss[0] == 0 and not grad.any()
