"""Rows whose logits are large against the temperature: the exponent of a logit is its difference to the largest one, however far
both are from zero."""
import numpy as np
import pytest
import torch

from logits_util import DTYPES, HALF_STEP, SMALLEST, sum_error
from oracle import logits as oracle

pytestmark = pytest.mark.gpu
F = np.float32
ROWS = 8


def bulks(dtype):
    """Where the rows' logits lie, with the temperature: |logit| / T from 2^20 to the end of the type's range."""
    if dtype == "fp16":
        return [(65504.0, 1e-5), (3001.0, 1e-6), (-65504.0, 1e-6), (-40000.0, 1e-3), (60000.0, 1.0), (-1000.0, 2.0)]
    far = [(1e7, 1.0), (-1e7, 2.0), (1e9, 1.0), (-1e9, 0.7), (1e10, 1.0), (-1e10, 2.0), (1e12, 1e6), (-1e15, 1e-3), (1e25, 1.0), (-1e25, 1e6), (1e29, 0.7),
           (3001.5, 1e-6), (-5000.0, 1e-6), (20.0, 1e-6), (3e38, 1e-6), (-3.3e38, 2.0)]
    return far


def rows_near(bulk, V, dtype, seed, T):
    """Rows around one value: a few steps of the type apart, differences of up to some 30 T, a masked part of it, ordinary logits behind
    a large negative stretch."""
    rng = np.random.default_rng(seed)
    t = DTYPES[dtype]
    z = np.full((ROWS, V), bulk)
    step = abs(bulk) * 2 * HALF_STEP[dtype]
    z[1] += step * rng.integers(-3, 4, V)
    z[2] += T * rng.uniform(-30, 0, V)
    z[3] += T * rng.normal(0, 3, V)
    z[4, rng.random(V) < 0.5] = -np.inf
    z[5, V // 3:] = rng.normal(0, 2, V - V // 3)
    z[6, :V - 5] = rng.normal(0, 2, V - 5) * T
    z[7] = np.where(np.arange(V) < V - 2, z[7], z[7] + np.abs(z[7]) * 0.5)
    limit = torch.finfo(t).max
    return torch.from_numpy(np.where(np.isfinite(z), np.clip(z, -limit, limit), z)).to(t)


@pytest.mark.parametrize("V", [900, 1500, 20001, 70001])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_log_sum_exp(dtype, V):
    import paper_1708_02983_amd as hip
    for n, (bulk, T) in enumerate(bulks(dtype)):
        z = rows_near(bulk, V, dtype, n, T)
        many = z.repeat(40 if V < 30000 else 1, 1)                       # whole rows a block each, too
        lse = hip.easgd_top_logits(many.cuda(), 5, temperature=T)[2].cpu().numpy().astype(np.float64)
        for r in range(len(many)):
            want = oracle.top_logits(z[r % ROWS].double().numpy(), 5, float(F(T)))[2]
            with np.errstate(over="ignore"):
                limit = np.float64(F(want))
            # one rounding of the result, and the sum's
            if np.isinf(limit):
                assert lse[r] == limit, (bulk, T, r, lse[r], want)
            else:
                assert abs(lse[r] - want) <= sum_error(V) + 2.0 ** -24 * abs(want), (bulk, T, r, lse[r], want)


@pytest.mark.parametrize("V, many", [(900, 1), (1500, 1), (20001, 1), (20001, 33), (70001, 1)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_loss_and_gradient(dtype, V, many):
    """All three ways to the exponentials of the cross-entropy: none of its own (hard 0, T 1), squares (T 2), one of its own."""
    import paper_1708_02983_amd as hip
    k = 6
    for n, (bulk, T) in enumerate(bulks(dtype)):
        hard = (0.0, 0.25, 0.5)[n % 3] if T not in (1.0, 2.0) else 0.5
        z = rows_near(bulk, V, dtype, 50 + n, T)
        T, hard = float(F(T)), float(F(hard))
        rng = np.random.default_rng(n)
        idx = np.stack([rng.choice(V, k, replace=False) for _ in range(ROWS)]).astype(np.int32)
        val = (rng.normal(0, 2.0, (ROWS, k)) * T).astype(F)
        z64 = z.double().numpy()
        labels = np.array([int(rng.choice(np.flatnonzero(z64[r] > -np.inf))) for r in range(ROWS)], np.int32)
        for r in range(ROWS):                                          # masked places would make the loss infinite
            idx[r] = rng.choice(np.flatnonzero(z64[r] > -np.inf), k, replace=False)
        rep = lambda a: torch.from_numpy(np.tile(a, (many,) + (1,) * (a.ndim - 1))).cuda()
        dev = z.repeat(many, 1).cuda()
        kw = dict(temperature=T, labels=rep(labels) if hard else None, hard=hard)
        up = min(64.0, 64.0 / T)
        both = hip.easgd_distill(dev, rep(idx), rep(val), scale=up, **kw)
        loss, state = hip.easgd_distill_loss(dev, rep(idx), rep(val), **kw)
        grad = hip.easgd_distill_grad(dev, rep(idx), rep(val), state, scale=up, **kw)
        up = float(F(up))
        ref = [oracle.distill(z64[r], idx[r], val[r], None, int(labels[r]) if hard else None, T, hard) for r in range(ROWS)]
        for l, g in (both, (loss, grad)):
            l, g = l.cpu().numpy().astype(np.float64), g.double().cpu().numpy()
            for r in range(many * ROWS):
                want, dz = ref[r % ROWS]
                row, eps = z64[r % ROWS], sum_error(V)
                with np.errstate(over="ignore"):
                    rounded = np.float64(F(want))
                # the logarithm of the sums moves by their relative error, 64-bit differences by 2^-52
                tol = (1 - hard) * T * T * 3 * eps + hard * eps + (2.0 ** -24 + 2.0 ** -50) * abs(want)
                if np.isinf(rounded):
                    assert l[r] == rounded, (bulk, T, r, l[r], want)
                else:
                    assert abs(l[r] - want) <= tol, (bulk, T, r, l[r], want)
                t = np.where(row > -np.inf, row.max() - row, 0.0)
                def q_tol(Tq):
                    q = np.exp(oracle.log_softmax(row, Tq))
                    return q * (2 * eps + 2.0 ** -24 * (6 + 3 * 1.4427 * t / Tq)) + 2.0 ** -126
                gt = up * ((1 - hard) * T * (q_tol(T) + 2.0 ** -23) + hard * (q_tol(1.0) + 2.0 ** -23))
                gt += HALF_STEP[dtype] * np.abs(dz * up) * 1.01 + 2.0 ** -24 * np.abs(dz * up) + SMALLEST[dtype]
                bad = ~(np.abs(g[r] - dz * up) <= gt)
                assert not bad.any(), (bulk, T, hard, r, np.flatnonzero(bad)[:4], g[r][bad][:4], (dz * up)[bad][:4])
