"""easgd_sample_tokens against the 64-bit oracle: the same tokens, and the logarithm of their probabilities."""
import numpy as np
import pytest
import torch

from logits_util import place
from oracle import logits as oracle

pytestmark = pytest.mark.gpu
F = np.float32
NEG = -np.inf


def check(z, dtype, u, temperature=None, top_k=None, top_p=None, min_p=None, pad=0, offset=0, exact_borders=False):
    import paper_1708_02983_amd as hip
    rows, V = z.shape
    dev, z64 = place(z, dtype, pad, offset)
    gpu = lambda a, t: None if a is None else torch.from_numpy(np.broadcast_to(np.asarray(a, t), (rows,)).copy()).cuda()
    tokens, logprob = hip.easgd_sample_tokens(dev, gpu(u, F), temperature=gpu(temperature, F), top_k=gpu(top_k, np.int32), top_p=gpu(top_p, F),
                                              min_p=gpu(min_p, F))
    torch.cuda.synchronize()
    tokens, logprob = tokens.cpu().numpy(), logprob.cpu().numpy().astype(np.float64)
    at = lambda a, r, default: default if a is None else float(np.broadcast_to(np.asarray(a, F), (rows,))[r])
    for r in range(rows):
        token, lp, gap = oracle.sample_token(z64[r], at(u, r, 0), at(temperature, r, 1.0), int(at(top_k, r, 0)), at(top_p, r, 1.0), at(min_p, r, 0.0))
        if not exact_borders:
            assert gap > 1e-8, f"row {r}: the drawn number sits on a border between two tokens, choose another seed"
        assert tokens[r] == token, (r, tokens[r], token)
        if token < 0:
            assert np.isnan(logprob[r])
        else:
            # one rounding to 32 bits; units of mass: V halves of a unit of 2^-(62 - log2 V) of the largest weight, at most
            assert abs(logprob[r] - lp) <= 2.0 ** -24 * abs(lp) + V * V * 2.0 ** -62 + 1e-12, (r, logprob[r], lp)


def draws(rng, rows):
    return rng.random(rows).astype(F)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows, V, pad, offset", [(1, 1, 0, 0), (7, 2, 1, 1), (40, 10, 0, 0), (33, 63, 0, 5), (20, 100, 0, 0), (9, 1000, 24, 0), (6, 1025, 0, 3),
                                                  (5, 4099, 0, 1), (6, 32000, 0, 0), (3, 50001, 0, 0), (2, 131072, 0, 0)])
def test_filters(dtype, rows, V, pad, offset):
    rng = np.random.default_rng(rows * 1000 + V)
    z = rng.normal(0, 2.0, (rows, V))
    z[:, :: max(1, V // 9)] += rng.uniform(2, 8, z[:, :: max(1, V // 9)].shape)
    T = rng.uniform(0.5, 1.5, rows)
    check(z, dtype, draws(rng, rows), pad=pad, offset=offset)
    check(z, dtype, draws(rng, rows), T, pad=pad, offset=offset)
    check(z, dtype, draws(rng, rows), T, top_k=rng.integers(0, min(V, 300) + 2, rows), pad=pad, offset=offset)
    check(z, dtype, draws(rng, rows), T, top_p=rng.uniform(0.3, 1.0, rows), pad=pad, offset=offset)
    check(z, dtype, draws(rng, rows), T, min_p=rng.uniform(0.0, 0.3, rows), pad=pad, offset=offset)
    check(z, dtype, draws(rng, rows), T, top_k=50, top_p=0.9, min_p=0.02, pad=pad, offset=offset)
    mixed = np.where(rng.random(rows) < 0.3, 0.0, T)
    check(z, dtype, draws(rng, rows), mixed, top_k=rng.choice([0, 1, 40, 5000, -3], rows), top_p=rng.choice([1.0, 0.5, 0.95, 2.0, 0.0], rows),
          min_p=rng.choice([0.0, 0.1, 1.0, 3.0, -1.0], rows), pad=pad, offset=offset)


@pytest.mark.parametrize("V", [1, 2, 64, 512, 4096, 65536])
def test_equal_logits_are_cut_exactly(V):
    """Equal logits: the token is floor(u * V) of those that are left, also where u * V is a whole number."""
    import paper_1708_02983_amd as hip
    u = np.unique(np.concatenate([np.arange(min(V, 64)) / min(V, 64), [1.0 - 2.0 ** -24, 0.3, 1.0, 7.0, -1.0, np.nan]]))
    rows = len(u)
    z = torch.full((rows, V), -7.25, device="cuda")
    du = torch.from_numpy(u.astype(F)).cuda()
    clean = np.clip(np.where(np.isnan(u), 0.0, u.astype(F)), 0.0, 1.0 - 2.0 ** -24)
    for top_k, n in ((None, V), (torch.full((rows,), max(1, V // 2), dtype=torch.int32, device="cuda"), max(1, V // 2))):
        tokens, logprob = hip.easgd_sample_tokens(z, du, top_k=top_k)
        np.testing.assert_array_equal(tokens.cpu().numpy(), np.floor(clean * n).astype(int))
        assert np.abs(logprob.cpu().numpy() + np.log(n)).max() <= 2.0 ** -24 * max(np.log(n), 1e-30) * 1.01
    if V >= 4:
        tokens, _ = hip.easgd_sample_tokens(z, du, top_p=torch.full((rows,), 0.5, device="cuda"))
        np.testing.assert_array_equal(tokens.cpu().numpy(), np.floor(clean * (V // 2)).astype(int))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [5, 700, 3000, 70001])
def test_ties_masks_and_special_values(dtype, V):
    rng = np.random.default_rng(V)
    z = np.stack([
        np.where(rng.random(V) < 0.5, 1.0, 2.0),
        rng.integers(-3, 4, V).astype(float),
        np.where(rng.random(V) < 20.0 / V, rng.normal(size=V), NEG),
        np.full(V, NEG),
        np.where(np.arange(V) == V // 2, 3.0, NEG),
        np.full(V, -3.3e38),
        np.where(np.arange(V) == V - 1, -1.0, -3.3e38),
        rng.normal(0, 1e37, V),
        rng.normal(0, 1e-39, V),
        np.linspace(-20, 20, V),
        np.where(np.arange(V) % 3 == 1, np.inf, 0.0),
        np.where(np.arange(V) == V // 3, np.nan, rng.normal(size=V)),
        np.full(V, np.nan),
        np.where(np.arange(V) % 2 == 0, -0.0, 0.0),
        rng.normal(0, 60.0, V),
        rng.normal(0, 0.01, V),
    ])
    rows = len(z)
    for n, (T, top_k, top_p, min_p) in enumerate(((None, None, None, None), (0.7, 30, None, None), (1.3, None, 0.8, None), (0.9, None, None, 0.05), (1.0, 1000, 0.7, 0.01),
                                                  (0.0, None, None, None), (np.inf, 3, None, None), (1e-30, None, 0.9, None), (np.nan, None, None, None))):
        u = np.random.default_rng(100 * n + V).random(rows) * 0.98 + 0.01
        check(z, dtype, u + 1e-4 * np.sqrt(2), T, top_k, top_p, min_p, pad=n % 3)


def test_every_token_in_proportion():
    """Stratified numbers over one distribution: token j is drawn n * p_j times, to one."""
    import paper_1708_02983_amd as hip
    n, V = 4096, 50
    z = np.random.default_rng(0).normal(0, 1.5, V).astype(F)
    u = torch.from_numpy(((np.arange(n) + 0.5) / n).astype(F)).cuda()
    tokens, _ = hip.easgd_sample_tokens(torch.from_numpy(z).cuda().expand(n, V).contiguous(), u)
    hits = np.bincount(tokens.cpu().numpy(), minlength=V)
    w = np.exp(z.astype(np.float64))
    assert np.abs(hits - n * w / w.sum()).max() <= 1.0 + 1e-6


def test_repeats_are_the_same():
    import paper_1708_02983_amd as hip
    for rows, V in ((600, 777), (64, 40000), (2, 200000)):
        z = torch.randn(rows, V, device="cuda").to(torch.bfloat16)
        u = torch.rand(rows, device="cuda")
        p = torch.full((rows,), 0.9, device="cuda")
        a = hip.easgd_sample_tokens(z, u, top_p=p)
        for _ in range(3):
            b = hip.easgd_sample_tokens(z, u, top_p=p)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    tokens, _ = hip.easgd_sample_tokens(z[:0], u[:0])
    assert tokens.shape == (0,)
