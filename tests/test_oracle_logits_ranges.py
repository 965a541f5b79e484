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
