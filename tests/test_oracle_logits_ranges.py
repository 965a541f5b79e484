"""The oracle of the calls on rows of logits where numbers are large, small or far apart."""
import numpy as np
import pytest

from oracle import logits as oracle


def test_differences_of_large_logits():
    """Logits that differ by units in 1e15: quotients by a temperature that is no power of two would lose the differences."""
    T = 0.7
    z = 1e15 + np.array([0.0, 1.0, 2.0])
    w = np.exp(np.arange(3) / T)
    assert np.allclose(oracle.log_softmax(z, T), np.log(w / w.sum()), rtol=0, atol=1e-14)
    assert oracle.logsumexp(z, T) == pytest.approx(1e15 / T + np.log(w.sum()), rel=1e-15)
    loss, grad = oracle.distill(z, [0], [0.0], temperature=T)
    assert loss == pytest.approx(-T * T * np.log(w[0] / w.sum()), abs=1e-13)
    assert np.allclose(grad, T * (w / w.sum() - [1, 0, 0]), rtol=0, atol=1e-14)


@pytest.mark.parametrize("gap", [10.0, 100.0, 600.0, 1e4, 1e9])
def test_rest_of_the_teacher_against_a_confident_student(gap):
    """One place at the gap, 999 others at 0, p = 0.9: 0.9 log(0.9 / q) + 0.1 log(0.1 / R), where R (1e-4342 at a gap of 1e4) is no 64-bit number."""
    z = np.zeros(1000)
    z[5] = gap
    log_all = gap + np.log1p(999 * np.exp(-gap))
    loss, grad = oracle.distill(z, [5], [np.log(0.9)], 0.0)
    assert loss == pytest.approx(0.9 * (np.log(0.9) - gap + log_all) + 0.1 * (np.log(0.1) - np.log(999) + log_all), rel=1e-12)
    q = np.exp(gap - log_all)
    want = np.full(1000, (1 - q) / 999 - 0.1 / 999)
    want[5] = q - 0.9
    assert np.allclose(grad, want, rtol=0, atol=1e-14)


def test_a_rest_without_a_place_counts_for_nothing():
    z = np.array([1.0, -np.inf, 2.0, -np.inf])
    loss, grad = oracle.distill(z, [0, 2], np.log([0.3, 0.4]), 0.0)
    lq = z[[0, 2]] - np.logaddexp(1.0, 2.0)
    assert loss == pytest.approx(0.3 * (np.log(0.3) - lq[0]) + 0.4 * (np.log(0.4) - lq[1]), abs=1e-15)
    assert np.allclose(grad, [0.7 * np.exp(lq[0]) - 0.3, 0, 0.7 * np.exp(lq[1]) - 0.4, 0], rtol=0, atol=1e-15)


def test_a_teacher_without_probability():
    """Masked values count for nothing, also against a log-sum-exp of -inf: the rest is 1, and the loss is -log R."""
    z = np.log([0.5, 0.25, 0.125, 0.125])
    with np.errstate(invalid="ignore"):
        for lse in (-np.inf, 0.3):
            loss, grad = oracle.distill(z, [0, 1], [-np.inf, -np.inf], lse)
            assert loss == pytest.approx(np.log(4)) and np.allclose(grad, [0.5, 0.25, 0.125 - 0.5, 0.125 - 0.5])
        loss, grad = oracle.distill(z, [0, 1], [-np.inf, -np.inf])
        assert loss == 0.0 and not grad.any()
        # values that differ by nothing at the end of fp32, and one that is all
        low = float(np.finfo(np.float32).min)
        loss, _ = oracle.distill(z, [0, 1], [low, low], temperature=1e-6)
        even, _ = oracle.distill(z, [0, 1], [0.0, 0.0], temperature=1e-6)
        assert loss == pytest.approx(even)
