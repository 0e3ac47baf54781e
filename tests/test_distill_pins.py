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


@pytest.mark.parametrize("gap", [1.0, 90.0, 700.0, 800.0, 1e5])
@pytest.mark.parametrize("T", [1.0, 0.1, 4.0])
def test_the_tail_far_below_the_list(gap, T):
    """Unlisted logits at -gap, -gap - T and -infinity next to listed ones at 0
    and -T: log p_rest = -gap / T + log(1 + 1/e) - log S, shares 1 : 1/e : 0."""
    e = np.exp(-1.0)
    x = np.array([[0.0, -gap, -T, -gap - T, -np.inf]])
    q, q_rest = np.array([0.6, 0.3]), 0.1
    loss, grad = S.distill_top(x, np.log(q)[None], np.array([[0, 2]]), T, True)
    S_top, rest = 1.0 + e, (1.0 + e) * np.exp(-gap / T)
    log_s = np.log(S_top + rest)
    log_rest = np.log(1.0 + e) - gap / T - log_s
    want = 0.6 * (np.log(0.6) + log_s) + 0.3 * (np.log(0.3) + 1.0 + log_s) + 0.1 * (np.log(0.1) - log_rest)
    assert abs(loss[0] - want) <= 1e-12 * max(1.0, abs(want))
    p = np.array([1.0, np.exp(-gap / T), e, np.exp(-gap / T) * e, 0.0]) / (S_top + rest)
    share = np.array([0.0, 1.0, 0.0, e, 0.0]) / (1.0 + e)
    assert np.abs(grad[0] - (p - [0.6, 0, 0.3, 0, 0] - q_rest * share) / T).max() < 1e-11 / T
    assert abs(grad.sum()) < 1e-12 / T
