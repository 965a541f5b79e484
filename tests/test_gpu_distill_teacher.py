"""A teacher's numbers at their ends: rows that the teacher masks as a whole, logits near the ends of fp32 at small temperatures."""
import numpy as np
import pytest
import torch

from logits_util import sum_error
from oracle import logits as oracle

pytestmark = pytest.mark.gpu
F = np.float32


def check(z, idx, val, lse, T):
    """All entry points; fp32 rows of ordinary logits, so that only the teacher's numbers can go wrong."""
    import paper_1708_02983_amd as hip
    rows, V = z.shape
    T = float(F(T))
    gpu = lambda a: None if a is None else torch.from_numpy(a).cuda()
    dev, kw = gpu(z), dict(temperature=T, teacher_lse=gpu(lse))
    both = hip.easgd_distill(dev, gpu(idx), gpu(val), **kw)
    loss, state = hip.easgd_distill_loss(dev, gpu(idx), gpu(val), **kw)
    split = loss, hip.easgd_distill_grad(dev, gpu(idx), gpu(val), state, **kw)
    for r in range(rows):
        want, dz = oracle.distill(z[r], idx[r], val[r], None if lse is None else np.float64(lse[r]), None, T)
        for l, g in (both, split):
            # the sums' relative error, twice (all places, those outside); the exponents of differences below 32 T; one rounding
            eps = 3 * sum_error(V) + 2.0 ** -24 * 100
            assert abs(l[r].item() - want) <= T * T * eps + 2.0 ** -24 * abs(want), (r, l[r].item(), want)
            assert np.abs(g[r].cpu().numpy() - dz).max() <= T * (eps + 2.0 ** -23) + 2.0 ** -24 * np.abs(dz).max(), r


LENGTHS = [40, 1000, 3000, 40000]


@pytest.mark.parametrize("V", LENGTHS)
def test_rows_that_the_teacher_masks(V):
    """Logits of -inf have probability 0 whatever the teacher's log-sum-exp is, -inf as easgd_top_logits writes it for such a row among them: all of
    the teacher's probability is its rest then."""
    rng = np.random.default_rng(V)
    rows, k = 5, 70
    z = rng.normal(0, 2.0, (rows, V)).astype(F)
    idx = np.stack([rng.permutation(max(V, k))[:k] for _ in range(rows)]).astype(np.int32)
    val = np.full((rows, k), -np.inf, F)
    lse = np.array([-np.inf, 0.5, -np.inf, 3e38, -np.inf], F)
    idx[2] = -1                                       # as easgd_top_logits writes it
    idx[4, ::2] = -1
    check(z, idx, val, lse, 1.0)
    check(z, idx, val, None, 1.0)
    val[1, 3] = val[3, 69] = 0.25
    check(z, idx, val, lse, 2.0)
    check(z, idx, val, None, 2.0)


def test_the_log_sum_exp_of_a_masked_row_goes_on():
    import paper_1708_02983_amd as hip
    t = torch.randn(3, 2000, device="cuda")
    t[1] = float("-inf")
    values, indices, lse = hip.easgd_top_logits(t, 8)
    z = torch.randn(3, 2000, device="cuda")
    for idx in (indices, indices.clamp(min=0)):
        loss, grad = hip.easgd_distill(z, idx, values, teacher_lse=lse)
        assert torch.isfinite(loss).all() and torch.isfinite(grad).all()


@pytest.mark.parametrize("V", LENGTHS)
@pytest.mark.parametrize("T", [0.5, 1e-3, 1e-6, 1.0])
def test_logits_at_the_ends_of_fp32(V, T):
    """Their quotients by a small temperature leave fp32; their differences count."""
    rng = np.random.default_rng(V + 1)
    rows, k = 6, 40
    z = (rng.normal(0, 2.0, (rows, V)) * T).astype(F)
    idx = np.stack([rng.permutation(V)[:k] for _ in range(rows)]).astype(np.int32)
    low = np.finfo(F).min
    val = np.full((rows, k), low, F)
    val[1] = -low
    val[2, 1:] = -low * F(0.5)
    val[3, 7] = 1.0
    val[4, :] = rng.normal(0, 1, k) * T
    val[4, 3] = low
    val[5, 10:] = -np.inf
    check(z, idx, val, None, T)
