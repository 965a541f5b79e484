"""The rest of the teacher's probability against students that put next to nothing outside its places: the logarithm of that mass is an
ordinary number long after the mass itself has left fp32, or 64 bits."""
import numpy as np
import pytest
import torch

from logits_util import DTYPES, HALF_STEP, SMALLEST, sum_error
from oracle import logits as oracle

pytestmark = pytest.mark.gpu
F = np.float32
GAPS = (20.0, 40.0, 46.0, 60.0, 80.0, 87.0, 88.5, 95.0, 100.0, 300.0, 600.0, 1e4, 6e4)


def students(V, dtype, seed):
    """A row for every gap: the teacher's places that far above all others, some of those masked; idx, val, lse [rows]."""
    rng = np.random.default_rng(seed)
    rows, k = len(GAPS), 4
    z = rng.normal(0, 0.5, (rows, V))
    idx = np.full((rows, k), -1, np.int32)
    for r, gap in enumerate(GAPS):
        idx[r, :3] = rng.choice(V, 3, replace=False)
        z[r, rng.random(V) < 0.1] = -np.inf
        z[r, idx[r, :3]] = gap + rng.normal(0, 0.5, 3)
        if r % 3 == 1:
            idx[r, 3] = idx[r, 0]
    val = rng.normal(2.0, 1.0, (rows, k)).astype(F)
    return torch.from_numpy(z).to(DTYPES[dtype]), idx, val


def check(z, idx, val, T, hard, dtype, many, scale, labels=None):
    import paper_1708_02983_amd as hip
    rows, V = z.shape
    T, hard, scale = float(F(T)), float(F(hard)), float(F(scale))
    z64 = z.double().numpy()
    used = idx >= 0
    lse = (np.log(np.where(used, np.exp(val.astype(np.float64) / T), 0.0).sum(axis=1)) + 0.1).astype(F)
    rep = lambda a: None if a is None else torch.from_numpy(np.tile(a, (many,) + (1,) * (a.ndim - 1))).cuda()
    dev = z.repeat(many, 1).cuda()
    kw = dict(temperature=T, teacher_lse=rep(lse), labels=rep(labels), hard=hard)
    both = hip.easgd_distill(dev, rep(idx), rep(val), scale=scale, **kw)
    loss, state = hip.easgd_distill_loss(dev, rep(idx), rep(val), **kw)
    dloss = torch.full((rows * many,), 0.5, device="cuda")
    grad = hip.easgd_distill_grad(dev, rep(idx), rep(val), state, dloss=dloss, scale=2 * scale, **kw)
    ref = [oracle.distill(z64[r], idx[r], val[r], np.float64(lse[r]), None if labels is None else int(labels[r]), T, hard) for r in range(rows)]
    eps = sum_error(V)
    for name, l, g in (("both", *both), ("split", loss, grad)):
        l, g = l.cpu().numpy().astype(np.float64), g.double().cpu().numpy()
        for r in range(rows * many):
            i = r % rows
            want, dz = ref[i]
            # sums: of all places and of those outside, each with its relative error; one rounding
            assert abs(l[r] - want) <= (1 - hard) * T * T * 3 * eps + hard * eps + 2.0 ** -24 * abs(want), (name, GAPS[i], r, l[r], want)
            row = z64[i]
            m = row.max()
            out = row > -np.inf
            out[idx[i][used[i]]] = False
            t = np.where(row > -np.inf, m - row, 0.0) / T * 1.4427
            q = np.exp(oracle.log_softmax(row, T))
            rest = max(0.0, 1.0 - oracle._teacher(V, idx[i], val[i], np.float64(lse[i]), T)[1].sum())
            share = np.zeros(V)
            if out.any():
                share[out] = np.exp(oracle.log_softmax(row[out], T))
            # a place's share of the mass outside: its exponent's roundings relative to the row's largest logit, twice (its own and the sum's),
            # and what is below the smallest normal number relative to a mass of 2^-64 at least
            far = float(t[out].min()) if out.any() else 0.0
            soft = q * (3 * eps + 2.0 ** -24 * (8 + 3 * t)) + rest * (share * (3 * eps + 2.0 ** -24 * (8 + 3 * t + 3 * min(far, 64.0))) + 2.0 ** -60)
            soft[idx[i][used[i]]] += 2.0 ** -22
            # (with rounding of the factor c - r / R, taken as a whole for places outside: one more of each part)
            soft += 2.0 ** -23 * (q + rest * share)
            ce = np.exp(oracle.log_softmax(row))
            gt = scale * ((1 - hard) * T * soft + hard * (ce * (2 * eps + 2.0 ** -24 * (8 + 3 * t * T)) + 2.0 ** -22))
            gt = gt * (1 + 2 * HALF_STEP[dtype]) + (HALF_STEP[dtype] + 2.0 ** -24) * np.abs(dz * scale) + SMALLEST[dtype]
            bad = ~(np.abs(g[r] - dz * scale) <= gt)
            assert not bad.any(), (name, GAPS[i], r, np.flatnonzero(bad)[:4], g[r][bad][:4], (dz * scale)[bad][:4], gt[bad][:4])


# wavefront rows, rows in parts, whole rows of each block
SHAPES = [(7, 1), (100, 1), (1000, 1), (1500, 1), (1500, 20), (20001, 1), (20001, 20), (70001, 20)]


@pytest.mark.parametrize("V, many", SHAPES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_confident_students(dtype, V, many):
    z, idx, val = students(V, dtype, V)
    rng = np.random.default_rng(V + 1)
    labels = rng.integers(0, V, len(GAPS)).astype(np.int32)
    z64 = z.double().numpy()
    for r in range(len(GAPS)):                                         # outside and inside the teacher's places, not masked
        labels[r] = idx[r, 0] if r % 2 else rng.choice(np.flatnonzero(z64[r] > -np.inf))
    for T, hard, scale in ((1.0, 0.0, 1024.0), (0.5, 0.0, 64.0), (2.0, 0.3, 64.0), (0.25, 0.5, 1024.0)):
        check(z, idx, val, T, hard, dtype, many, scale, labels if hard else None)


@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_finite_masks(V):
    """A vocabulary that is masked with a large finite number outside the teacher's places."""
    z, idx, val = students(V, "fp32", 3)
    masks = [-1e4, -1e9, -3e38, -65504.0, -1e10, -1e20, -1e30, -50.0, -100.0, -200.0, -1e3, -1e5, -1e6]
    for r, mask in enumerate(masks):
        keep = z[r, torch.from_numpy(idx[r, :3]).long()].clone() - GAPS[r]
        z[r] = mask
        z[r, torch.from_numpy(idx[r, :3]).long()] = keep
    check(z, idx, val, 1.0, 0.0, "fp32", 1, 8.0)
    check(z, idx, val, 0.5, 0.0, "fp32", 25 if V > 3000 else 1, 8.0)


@pytest.mark.parametrize("V, many", SHAPES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_few_places_in_masked_rows(dtype, V, many):
    """Nearly all of a row is masked with -inf: one logit outside the teacher's places far below them (beside one of them, at either end, or
    none at all), and outside logits that come before the ones that dwarf them."""
    rows = len(GAPS)
    rng = np.random.default_rng(V)
    z = np.full((rows, V), -np.inf)
    idx = np.full((rows, 4), -1, np.int32)
    val = rng.normal(2.0, 1.0, (rows, 4)).astype(F)
    for r in range(rows):
        idx[r, :3] = V - 1 - rng.permutation(min(V, 40) - 1)[:3] if r % 2 else 1 + rng.permutation(min(V, 40) - 1)[:3]
        free = np.setdiff1d(np.arange(V), idx[r, :3])
        where = (free[0], free[-1], free[np.argmin(np.abs(free - idx[r, 0]))], None)[r % 4]
        z[r, idx[r, :3]] = rng.normal(0, 1, 3)
        if where is not None:
            z[r, where] = -500.0 if r < 8 else -90.0
        if r >= 9:
            z[r, free[:max(1, V // 3)]] = -400.0 + rng.normal(0, 1, max(1, V // 3))
    check(torch.from_numpy(z).to(DTYPES[dtype]), idx, val, 1.0, 0.0, dtype, many, 16.0)
    check(torch.from_numpy(z).to(DTYPES[dtype]), idx, val, 0.5, 0.0, dtype, many, 16.0)


def test_the_place_that_is_all():
    """One place at 100, the others at 0: loss 0.9 log 0.9 + 0.1 log(0.1 / 999) + 0.1 * 100, as worked out by hand."""
    import paper_1708_02983_amd as hip
    z = torch.zeros(1, 1000, device="cuda")
    z[0, 5] = 100.0
    idx, val = torch.tensor([[5]], dtype=torch.int32, device="cuda"), torch.tensor([[float(np.log(0.9))]], device="cuda")
    loss, grad = hip.easgd_distill(z, idx, val, teacher_lse=torch.zeros(1, device="cuda"))
    want = 0.9 * np.log(0.9) + 0.1 * np.log(0.1 / 999) + 10.0
    assert abs(loss.item() - want) <= 1e-5
    assert abs(grad[0, 5].item() - 0.1) <= 1e-6 and (grad[0, :5] + 0.1 / 999).abs().max().item() <= 1e-9
