"""The oracle of given tokens against hand values, differences and other ways to compute the same."""
import numpy as np
import pytest

from oracle import tokens as ot

rng = np.random.default_rng(5)


def test_hand_values():
    z = np.log([0.5, 0.25, 0.125, 0.125])
    lp, h, rank, top, places = ot.score(z, 2, k=3)
    assert np.isclose(lp, np.log(0.125)) and np.isclose(h, 1.75 * np.log(2)) and rank == 2
    assert places.tolist() == [0, 1, 2] and np.allclose(np.exp(top), [0.5, 0.25, 0.125])
    assert ot.score(z, 3)[2] == 3                                        # equal logits: by index
    assert ot.score(z, 4)[:3] == (0.0, 0.0, -1) and ot.score(z, -1)[:3] == (0.0, 0.0, -1)
    assert ot.score([5.0], 0)[:3] == (0.0, 0.0, 0)


def test_masked_places():
    z = np.array([0.0, -np.inf, 0.0, -np.inf])
    lp, h, rank, top, places = ot.score(z, 1, k=3)
    assert lp == -np.inf and np.isclose(h, np.log(2)) and rank == 2 and places.tolist() == [0, 2, -1] and top[2] == -np.inf
    none = np.full(3, -np.inf)
    assert ot.score(none, 1)[:3] == (-np.inf, 0.0, 0) and not ot.score_grad(none, 1, 1.0, 1.0, 1.0).any()
    assert ot.token_loss(none, 1)[0] == 0.0
    assert np.isnan(ot.score([0.0, np.inf, 1.0], 0)[:2]).all() and ot.score([0.0, np.inf, 1.0], 2)[2] == 1
    assert np.isnan(ot.score([0.0, np.nan, 1.0], 0)[:2]).all()


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_gradient_against_differences(T):
    z = rng.normal(size=23) * 2
    z[4] = -np.inf
    token, a, b = 7, 1.3, -0.4
    f = lambda x: a * ot.score(x, token, T)[0] + b * ot.score(x, token, T)[1]
    d = ot.score_grad(z, token, T, a, b)
    for j in range(23):
        if j == 4:
            continue
        up, down = z.copy(), z.copy()
        up[j] += 1e-5
        down[j] -= 1e-5
        assert np.isclose((f(up) - f(down)) / 2e-5, d[j], rtol=1e-6, atol=1e-9)
    loss, grad = ot.token_loss(z, token, -a, -b, T)
    assert np.isclose(loss, f(z)) and np.allclose(grad, d)
