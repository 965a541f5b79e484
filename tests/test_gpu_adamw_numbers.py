"""AdamW rounds at the ends of the numbers' ranges: gradients of 0 where eps is small and the rate large."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def hip():
    import paper_1708_02983_amd as pkg
    return pkg


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
