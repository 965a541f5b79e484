"""easgd_grad_token_loss of networks whose product of logits is cut along its sum (a last layer of 128 inputs and more): partial logits are added up row by row
before they are scored."""
import numpy as np
import pytest
import torch

from gpu_util import normwise, to_dev, to_host
from oracle import tokens as ot
from test_gpu_logits_calls import forward, gradient, network
from test_gpu_score import bounds

pytestmark = pytest.mark.gpu
F = np.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def hip():
    import paper_1708_02983_amd as pkg
    return pkg


def logit_error(dims, w, X):
    """How far the logits of a worker may be off: a sum of K products of 32 bits, each rounded and added in some order, by (K + 1) 2^-24 of the products'
    magnitudes, and what the layer below is off by, through the magnitudes of the weights."""
    a, off = np.abs(X.astype(np.float64)), np.zeros(X.shape)
    acts, _, _ = forward(dims, w, X)
    at = 0
    for l in range(len(dims) - 1):
        wl = np.abs(w[at:at + dims[l] * dims[l + 1]].astype(np.float64)).reshape(dims[l], dims[l + 1])
        bias = np.abs(w[at + dims[l] * dims[l + 1]:at + (dims[l] + 1) * dims[l + 1]].astype(np.float64))
        off = (dims[l] + 2) * U * (np.abs(acts[l]) @ wl + bias) + off @ wl
        at += (dims[l] + 1) * dims[l + 1]
    return off


@pytest.mark.parametrize("dims, P, b, bonus, T, weighted, seed", [
    ((784, 10), 3, 7, 0.0, 1.0, True, 1),               # seven parts, a wavefront's two registers
    ((784, 10), 1, 1, 0.5, 2.0, False, 2),
    ((784, 1000), 2, 5, 0.25, 0.5, True, 3),            # seven parts, sixteen registers
    ((50, 300, 100), 4, 6, 0.1, 1.0, True, 4),          # three parts
    ((40, 1024, 1000), 2, 4, 0.25, 1.5, True, 8),       # nine parts
    ((30, 128, 129), 2, 5, 0.0, 1.0, True, 6),          # two, the second with the bias alone
    ((2100, 7), 2, 3, 0.1, 1.0, False, 7)])             # the most parts, sixteen
def test_logits_that_come_in_parts(hip, dims, P, b, bonus, T, weighted, seed):
    N, ld, W, X, y = network(dims, P, b, seed)
    rng = np.random.default_rng(seed)
    tokens = y.astype(np.int32)
    if b > 3:
        tokens[0, 2], tokens[P - 1, b - 1] = -1, dims[-1]       # padding at either end of the classes
        tokens[P - 1, 0] = dims[-1] - 1
    weight = rng.normal(size=(P, b)).astype(F) if weighted else None
    G = torch.full((P, ld), float("nan"), device="cuda")
    loss, logprob, entropy = torch.empty(P, device="cuda"), torch.empty(P, b, device="cuda"), torch.empty(P, b, device="cuda")
    call = lambda: hip.easgd_grad_token_loss(dims, to_dev(W), to_dev(X), to_dev(tokens), G, loss=loss, weight=None if weight is None else to_dev(weight), bonus=bonus,
                                             temperature=T, logprob=logprob, entropy=entropy)
    call()
    first = G.clone()
    ref = np.full((P, ld), np.nan)
    for p in range(P):
        _, z, near = forward(dims, W[p], X[p])
        assert near > 1e-5, "a hidden unit within rounding of zero: choose another seed"
        off = logit_error(dims, W[p], X[p]).max(axis=1) / T
        dz, total, may = np.zeros_like(z), 0.0, 0.0
        for r in range(b):
            token, w = int(tokens[p, r]), 1.0 if weight is None else float(weight[p, r])
            l, g = ot.token_loss(z[r], token, w, float(F(bonus)), T)
            dz[r], total = g / b, total + l
            lp, h, *_ = ot.score(z[r], token, T)
            # a log probability moves by twice what the logits do at most, an entropy by its slope, |log q + H| q, whose sum is 2 H at most; then the row's own sums
            e_lp, e_h = bounds(z[r], token, T)
            e_lp, e_h = e_lp + 2 * off[r] + U * abs(lp), e_h + 2 * h * off[r] * (1 + off[r])
            assert abs(logprob[p, r].item() - lp) <= e_lp and abs(entropy[p, r].item() - h) <= e_h, (p, r)
            may += abs(w) * e_lp + bonus * e_h
        ref[p, :N] = gradient(dims, W[p], X[p], dz)
        assert abs(loss[p].item() - total / b) <= may / b + 2.0 ** -20 * abs(total / b)
    assert normwise(to_host(G), ref) <= 1e-5
    call()
    assert torch.equal(G[:, :N], first[:, :N]), "not the same from run to run"
