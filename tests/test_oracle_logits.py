"""The oracle of the calls on rows of logits, pinned by closed forms, brute force and differences."""
import itertools

import numpy as np
import pytest

from oracle import logits as oracle


def test_order_and_top():
    z = [1.0, -np.inf, 3.0, 0.0, 3.0, -0.0, np.nan]
    assert oracle.order(z).tolist() == [2, 4, 0, 3, 5]
    values, indices, lse = oracle.top_logits(z[:6], 7)
    assert indices.tolist() == [2, 4, 0, 3, 5, -1, -1]
    assert values.tolist() == [3.0, 3.0, 1.0, 0.0, 0.0, -np.inf, -np.inf]
    assert lse == pytest.approx(np.log(2 * np.e ** 3 + np.e + 2), abs=1e-14)
    assert oracle.top_logits([0.0] * 8, 2, 5.0)[2] == pytest.approx(np.log(8), abs=1e-15)
    assert oracle.top_logits([-np.inf] * 3, 1)[2] == -np.inf
    assert oracle.top_logits([0.0, np.inf], 1)[2] == np.inf
    assert np.isnan(oracle.top_logits([0.0, np.nan], 1)[2])


def test_loss_closed_forms():
    # a student that is the teacher: 0, with every place named or the rest as one more outcome
    z = np.log([0.5, 0.25, 0.125, 0.125])
    for lse in (None, 0.0):
        loss, grad = oracle.distill(z, [2, 0, 1, 3], z[[2, 0, 1, 3]], lse)
        assert abs(loss) < 1e-15 and np.abs(grad).max() < 1e-15
    loss, grad = oracle.distill(z, [0, 1], z[:2], 0.0)
    assert abs(loss) < 1e-15 and np.abs(grad).max() < 1e-15
    # one place, all of the teacher's probability: the cross-entropy of that place
    loss, grad = oracle.distill(z, [1], [7.0])
    assert loss == pytest.approx(np.log(4)) and np.allclose(grad, [0.5, -0.75, 0.125, 0.125])
    hard, _ = oracle.distill(z, [1], [7.0], label=1, hard=1.0)
    assert hard == pytest.approx(np.log(4))
    # the temperature: T^2 KL of the softened distributions
    loss, _ = oracle.distill([0.0, 2.0], [0, 1], [2.0, 0.0], temperature=2.0)
    p = 1 / (1 + np.exp(-1.0))
    assert loss == pytest.approx(4 * (p - (1 - p)) * 1.0)
    # the same place twice counts with both probabilities; unused slots do not count
    a = oracle.distill(z, [1, 1, -1, 9], [0.0, 0.0, 50.0, 50.0])
    b = oracle.distill(z, [1], [0.0])
    assert a[0] == pytest.approx(b[0] - np.log(2)) and np.allclose(a[1], b[1])
    # what counts as nothing
    for row in (oracle.distill(z, [0], [0.0], label=-1), oracle.distill(z, [0], [0.0], label=4), oracle.distill([-np.inf] * 4, [0], [0.0]),
                oracle.distill(z, [-1, 4], [0.0, 0.0]), oracle.distill(z, [-1, -1], [0.0, 0.0], 1.0), oracle.distill(z, [2], [-np.inf])):
        assert row[0] == pytest.approx(0.0, abs=1e-15) and np.abs(row[1]).max() < 1e-15
    assert oracle.distill([0.0, -np.inf], [1], [0.0])[0] == np.inf
    assert np.allclose(oracle.distill([0.0, -np.inf], [1], [0.0])[1], [1.0, -1.0])


@pytest.mark.parametrize("tail, hard, T", itertools.product((False, True), (0.0, 0.3, 1.0), (1.0, 2.5)))
def test_gradient_against_differences(tail, hard, T):
    rng = np.random.default_rng(5)
    V, k = 13, 5
    z, a = rng.normal(0, 2, V), rng.normal(1, 2, k)
    idx = np.array([3, 11, 3, 0, -1])
    lse = oracle.logsumexp(a[:4] / T) + 0.2 if tail else None
    label = 7
    loss = lambda x: oracle.distill(x, idx, a, lse, label, T, hard)[0]
    grad = oracle.distill(z, idx, a, lse, label, T, hard)[1]
    for j in range(V):
        e = np.zeros(V); e[j] = 1e-5
        assert (loss(z + e) - loss(z - e)) / 2e-5 == pytest.approx(grad[j], abs=1e-8)


def test_sampling_closed_forms():
    # equal logits: the token is floor(u * V); ties are cut by ascending index
    for V in (1, 2, 8):
        for i in range(2 * V):
            assert oracle.sample_token(np.zeros(V), (i + 0.5) / (2 * V))[0] == i // 2
    assert oracle.sample_token(np.zeros(8), 0.99, top_k=3)[0] == 2
    assert oracle.sample_token(np.zeros(8), 0.99, top_p=0.5)[0] == 3
    assert oracle.sample_token(np.zeros(8), 0.99, top_p=0.51)[0] == 4
    z = np.log([0.1, 0.4, 0.2, 0.3])
    assert [oracle.sample_token(z, u)[0] for u in (0.05, 0.15, 0.65, 0.75)] == [0, 1, 2, 3]
    assert oracle.sample_token(z, 0.9, min_p=0.6)[0] == 3 and oracle.sample_token(z, 0.5, min_p=0.6)[0] == 1
    assert oracle.sample_token(z, 0.9, min_p=0.8)[0] == 1
    assert oracle.sample_token(z, 0.99, top_k=3, top_p=0.75)[0] == 3          # 0.4 + 0.3 of 0.9 reach it
    assert oracle.sample_token(z, 0.99, top_p=0.0)[0] == 1
    assert oracle.sample_token(z, 0.7, temperature=0.0)[:2] == (1, 0.0)
    token, logprob, _ = oracle.sample_token(z, 0.75, top_k=2)
    assert token == 3 and logprob == pytest.approx(np.log(3 / 7))
    # masks
    assert oracle.sample_token([-np.inf] * 3, 0.5)[0] == -1
    assert oracle.sample_token([-np.inf, 0.0, np.nan], 0.99)[0] == 1
    assert oracle.sample_token([np.inf, 5.0, np.inf], 0.6)[0] == 2


def test_sampling_frequencies():
    """Stratified numbers hit every token in proportion to its probability."""
    z = np.array([0.3, -1.0, 2.0, 0.3, 1.0])
    n = 20000
    hits = np.bincount([oracle.sample_token(z, (i + 0.5) / n, temperature=0.7, top_k=4)[0] for i in range(n)], minlength=5) / n
    w = np.exp(z / 0.7); w[1] = 0.0
    assert np.abs(hits - w / w.sum()).max() < 1e-3
