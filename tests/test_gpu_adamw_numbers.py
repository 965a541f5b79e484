"""AdamW rounds at the ends of the numbers' ranges: second moments below the normal numbers, and gradients of 0 where eps is small and the rate large."""
import numpy as np
import pytest
import torch

from oracle import adamw as oa

pytestmark = pytest.mark.gpu
F = np.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def hip():
    import paper_1708_02983_amd as pkg
    return pkg


@pytest.mark.parametrize("low,high", [(-149, -140), (-149, -126), (-130, -100), (-149, -60)])
def test_roots_of_the_smallest_second_moments(hip, low, high):
    """The roots' own S is what the oracle takes them of (the kernel's bits), so nothing here is left out of the comparison: a parameter of 0 moves by the
    quotient alone, whose sixteen roundings are those of every other."""
    P, N = 3, 1000
    rng = np.random.default_rng(-low)
    S = np.exp2(rng.uniform(low, high, (P, N))).astype(F)
    S[0, :200] = np.exp2(np.arange(200) % (high - low + 1) + low).astype(F)         # powers of two, the smallest among them
    M = (rng.normal(size=(P, N)) * np.sqrt(S.astype(np.float64))).astype(F)
    W, G = np.zeros((P, N), F), np.zeros((P, N), F)
    for eps in (1e-30, 1e-25):
        dW, dM, dS = (torch.from_numpy(x).cuda() for x in (W, M, S))
        hip.adamw_round(dW, dM, dS, torch.from_numpy(G).cuda(), 3, 0.01, beta1=0.5, beta2=0.75, eps=eps, decay=0.0)
        want, _, M1, S1, size = oa.adamw_round(W, M, S, G, None, 3, 0.01, beta1=0.5, beta2=0.75, eps=eps, decay=0.0)
        assert np.array_equal(dM.cpu().numpy(), M1) and np.array_equal(dS.cpu().numpy(), S1)
        assert (S1 < 2.0 ** -60).all() and ((0 < S1) & (S1 < 2.0 ** -100)).sum() > N
        off = np.abs(dW.double().cpu().numpy() - want) - U * (np.abs(want) + 16 * size) - 1e-45
        assert (off <= 0).all(), (int(off.argmax()), off.max())


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("N", [600, 64 * 256 * 256 + 300])
@pytest.mark.parametrize("center", [False, True])
def test_gradients_of_zero_with_a_small_eps_and_a_large_rate(hip, eight, N, center):
    """0 / (0 + eps) is 0 whatever the rate is: a parameter that has never had a gradient moves by its decay alone.  eta / ((1 - beta1) eps) is above what 32 bits hold."""
    P, eta, decay = 2, 1e9, 0.5e-9
    W = torch.ones((P, N), device="cuda")
    Wc = torch.ones((N,), device="cuda") if center else None
    if eight:
        M, S = torch.zeros((P, N), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.zeros((P, N), dtype=torch.uint8, device="cuda").view(torch.float8_e5m2)
        more = dict(M_scale=torch.zeros((P, (N + 255) // 256), device="cuda"), S_scale=torch.zeros((P, (N + 255) // 256), device="cuda"))
    else:
        M, S, more = torch.zeros((P, N), device="cuda"), torch.zeros((P, N), device="cuda"), {}
    hip.adamw_round(W, M, S, torch.zeros((P, N), device="cuda"), 1, eta, Wc=Wc, eps=1e-30, decay=decay, **more)
    # the rate times the decay is one rounding, and so is either of them
    want = 1.0 - eta * decay
    assert ((W.double() - want).abs() <= 4 * U).all(), W[0, 0].item()
