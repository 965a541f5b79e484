"""easgd_distill, easgd_distill_loss, easgd_distill_grad against the 64-bit oracle and against differences."""
import itertools

import numpy as np
import pytest
import torch

from logits_util import DTYPES, HALF_STEP, SMALLEST, place, sum_error
from oracle import logits as oracle

pytestmark = pytest.mark.gpu
F = np.float32


def teacher(rng, rows, V, k, T, twice=False, unused=True):
    """Teacher's slots: some not used, some naming the same place where asked for."""
    idx = np.full((rows, k), -1, np.int32)
    for r in range(rows):
        n = min(k, V)
        idx[r, :n] = rng.choice(V, n, replace=False)
        if unused and n > 2:
            idx[r, rng.integers(0, n)] = V + 5 if r % 2 else -7
        if twice and n > 3:
            idx[r, n - 1] = idx[r, 0]
    val = rng.normal(3.0, 2.0, (rows, k)).astype(F)
    used = (idx >= 0) & (idx < V)
    a = np.where(used, val.astype(np.float64) / T, -np.inf)
    with np.errstate(divide="ignore"):
        lse = np.log(np.exp(a).sum(axis=1)) + rng.uniform(0.01, 0.5, rows)
    return idx, val, np.where(np.isfinite(lse), lse, 0.0).astype(F)


def bounds(z, idx, val, lse, label, T, hard, up, dtype):
    """How far loss and gradient of one row may be off: the sums' relative error moves log sum by as much and every q by as
    much; an element's own exponent carries three roundings of |t| and the exponential and the two products five more."""
    V = len(z)
    eps = sum_error(V)
    if not (z > -np.inf).any():
        return 0.0, np.zeros(V)                       # nothing to learn: exactly 0
    loss_tol = (1 - hard) * T * T * 1.5 * eps * 2 + hard * eps + 1e-12
    m = np.max(z[z > -np.inf], initial=-np.inf)
    t = np.where(z > -np.inf, (m - z), 0.0)
    def q_tol(Tq):
        q = np.exp(oracle.log_softmax(z / Tq))
        return q * (2 * eps + 2.0 ** -24 * (6 + 2.1 * t / Tq * 1.4427))
    soft = q_tol(T)
    used, p, _, target = oracle._teacher(V, idx, val, lse, T)
    if lse is not None:
        outside = np.ones(V, bool); outside[idx[used]] = False
        R = np.exp(oracle.log_softmax(z / T))[outside].sum()
        r = max(0.0, 1 - p.sum())
        if R > 0:
            soft = soft * (1 + 2 * r / R)
    grad_tol = abs(up) * ((1 - hard) * T * (soft + 2.0 ** -23 * target) + hard * (q_tol(1.0) + 2.0 ** -23))
    return loss_tol, grad_tol


def check(z, idx, val, lse, labels, T, hard, dtype, pad=0, offset=0, scale=1.0, dloss=None, dpad=0, doffset=0, entries=("both", "split")):
    import paper_1708_02983_amd as hip
    rows, V = z.shape
    T = float(F(T)); hard = float(F(hard)); scale = float(F(scale))
    dev, z64 = place(z, dtype, pad, offset)
    gpu = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    args = dict(temperature=T, teacher_lse=gpu(lse), labels=gpu(labels), hard=hard)
    idx_d, val_d = gpu(idx), gpu(val)
    results = []
    for entry in entries:
        dl, _ = place(np.full((rows, V), 777.0), dtype, dpad, doffset)
        if entry == "both":
            loss, grad = hip.easgd_distill(dev, idx_d, val_d, scale=scale, dlogits=dl, **args)
            up = np.full(rows, scale)
        else:
            loss, state = hip.easgd_distill_loss(dev, idx_d, val_d, **args)
            grad = hip.easgd_distill_grad(dev, idx_d, val_d, state, scale=scale, dloss=gpu(dloss), dlogits=dl, **args)
            up = scale * (np.ones(rows) if dloss is None else dloss.astype(np.float64))
        torch.cuda.synchronize()
        base = dl._base if dl._base is not None else dl
        assert torch.isnan(base[:doffset]).all()
        if dpad:                                     # what lies between the rows is as it was
            whole = base[doffset:doffset + rows * (V + dpad)].view(rows, V + dpad)
            assert torch.isnan(whole[:, V:]).all()
        results.append((entry, loss.cpu().numpy().astype(np.float64), grad.double().cpu().numpy(), up))
    for r in range(rows):
        label = None if labels is None else int(labels[r])
        l_ref, g_ref = oracle.distill(z64[r], idx[r], val[r], None if lse is None else np.float64(lse[r]), label, T, hard)
        lt = gt = None
        if label is None or 0 <= label < V:
            lt, gt = bounds(z64[r], idx[r], val[r].astype(np.float64), None if lse is None else np.float64(lse[r]), label, T, hard, 1.0, dtype)
        for entry, loss, grad, up in results:
            if lt is None:
                assert loss[r] == 0.0 and not grad[r].any(), (entry, r)
                continue
            if abs(l_ref) > np.finfo(F).max:           # a loss is 32 bits: beyond the largest one it is infinite
                l_ref = np.sign(l_ref) * np.inf
            if np.isfinite(l_ref):
                assert abs(loss[r] - l_ref) <= lt + 2.0 ** -24 * abs(l_ref), (entry, r, loss[r], l_ref, lt)
            else:
                np.testing.assert_array_equal(loss[r], l_ref)
            g = g_ref * up[r]
            tol = gt * abs(up[r]) + HALF_STEP[dtype] * (np.abs(g) + gt * abs(up[r])) + 2.0 ** -24 * np.abs(g) + SMALLEST[dtype] * (1 + abs(up[r]))
            bad = ~(np.abs(grad[r] - g) <= tol)
            assert not bad.any(), (entry, r, np.flatnonzero(bad)[:5], grad[r][bad][:5], g[bad][:5], tol[bad][:5])


SIZES = [(1, 1, 1), (3, 2, 4), (5, 7, 3), (130, 10, 10), (70, 100, 10), (9, 64, 64), (6, 255, 256), (33, 1000, 10), (5, 1024, 100), (5, 1025, 33),
         (7, 4099, 256), (3, 32000, 64), (2, 50001, 20), (1, 131072, 64)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows, V, k", SIZES)
def test_sizes(dtype, rows, V, k):
    rng = np.random.default_rng(V * 7 + k)
    z = rng.normal(0, 2.0, (rows, V))
    for n, (tail, hard) in enumerate(((False, 0.0), (True, 0.0), (False, 0.4), (True, 0.25), (False, 1.0))):
        T = (1.0, 2.0, 0.7)[n % 3]
        idx, val, lse = teacher(rng, rows, V, k, T, twice=n == 2)
        labels = rng.integers(-1, V, rows).astype(np.int32) if hard else None
        # gradients large enough for 16 bits to hold them
        check(z, idx, val, lse if tail else None, labels, T, hard, dtype, pad=n, offset=n, scale=64.0,
              dloss=rng.uniform(0.5, 2.0, rows).astype(F), dpad=(0, 3, 0, 1, 0)[n], doffset=(0, 1, 2, 0, 5)[n])


@pytest.mark.parametrize("V, k", [(10, 256), (100, 256), (900, 200), (1024, 65), (1500, 256), (40000, 130)])
def test_places_named_many_times(V, k):
    """Places drawn with repetition from few and from all; one place in every slot; between slots that are not used."""
    rng = np.random.default_rng(V + k)
    rows, T = 6, 2.0
    z = rng.normal(0, 2.0, (rows, V))
    idx = rng.integers(0, V, (rows, k)).astype(np.int32)
    idx[1] = rng.integers(0, min(V, 7), k)
    idx[2] = V - 1
    idx[3, ::2] = -1
    idx[4] = np.where(np.arange(k) % 64 == 63, 3, V)
    idx[5] = idx[5, ::-1] // 2
    val = rng.normal(0.0, 2.0, (rows, k)).astype(F)
    used = (idx >= 0) & (idx < V)
    lse = (np.log(np.where(used, np.exp(val.astype(np.float64) / T), 0.0).sum(axis=1)) + 0.25).astype(F)
    labels = rng.integers(0, V, rows).astype(np.int32)
    labels[2] = V - 1
    for tail, hard in ((False, 0.0), (True, 0.3)):
        check(z, idx, val, lse if tail else None, labels if hard else None, T, hard, "fp32", scale=4.0)


@pytest.mark.parametrize("V, rows", [(262144, 2), (1048576, 1)])
def test_longest_rows(V, rows):
    rng = np.random.default_rng(1)
    z = rng.normal(0, 2.0, (rows, V))
    idx, val, lse = teacher(rng, rows, V, 256, 1.0)
    check(z, idx, val, lse, None, 1.0, 0.0, "bf16", offset=1, scale=1024.0)
    check(z, idx, val, None, np.array([5, -1][:rows], np.int32), 2.0, 0.5, "fp32", offset=1)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [6, 600, 5000])
def test_masked_places(dtype, V):
    """Masked logits, a row with none left, a teacher whose place the student has masked, a teacher without slots, one with
    masked values, all places named."""
    rng = np.random.default_rng(V)
    z = rng.normal(0, 2.0, (8, V))
    z[0, rng.random(V) < 0.5] = -np.inf
    z[0, 0] = 1.0
    z[1] = -np.inf
    z[2] = -3.3e38
    z[3, 1:] = -np.inf
    z[5] = np.where(np.arange(V) % 3 == 0, -3.3e38, z[5])
    idx, val, lse = teacher(rng, 8, V, 6, 1.0, unused=False)
    idx[0, 0] = 0; idx[0, 1:] = -1                    # the one place is there
    idx[3] = [0, -1, -1, -1, -1, -1]
    idx[4] = -1
    val[5, 2:] = -np.inf
    val[6] = -np.inf
    for tail, labels in itertools.product((False, True), (None, np.array([0, 1, 2, 0, 3, 4, -1, V], np.int32))):
        check(z, idx, val, lse if tail else None, labels, 1.5, 0.0 if labels is None else 0.5, dtype, pad=1)
    # a place that the student masks: an infinite loss, a finite gradient
    z[3, 2] = 0.5
    idx[3, 1] = 4
    check(z, idx, val, None, None, 1.0, 0.0, dtype)


def test_not_a_number_stays_in_its_row():
    import paper_1708_02983_amd as hip
    z = torch.randn(3, 2000, device="cuda")
    z[1, 77] = float("nan")
    idx = torch.arange(8, dtype=torch.int32, device="cuda").repeat(3, 1)
    val = torch.randn(3, 8, device="cuda")
    loss, grad = hip.easgd_distill(z, idx, val)
    assert torch.isnan(loss).tolist() == [False, True, False]
    assert torch.isnan(grad[1]).all() and torch.isfinite(grad[0]).all() and torch.isfinite(grad[2]).all()


def test_gradient_against_differences_of_the_losses():
    """Central differences of the kernel's own forward pass: the step moves the loss by about 1e-2 of a gradient entry's size,
    whose third-order term and the losses' rounding (2^-24 of a loss near 3, over 2e-2) stay below 1e-4."""
    import paper_1708_02983_amd as hip
    rng = np.random.default_rng(3)
    V, k = 40, 6
    z = rng.normal(0, 1.0, V).astype(F)
    idx, val, lse = teacher(rng, 1, V, k, 1.0)
    gpu = lambda a: torch.from_numpy(a).cuda()
    label = np.array([9], np.int32)
    step = 1e-2
    many = np.concatenate([z + step * np.eye(V, dtype=F), z - step * np.eye(V, dtype=F)])
    rep = lambda a: gpu(np.repeat(a, 2 * V, axis=0))
    loss, _ = hip.easgd_distill_loss(gpu(many), rep(idx), rep(val), teacher_lse=rep(lse), labels=rep(label), hard=0.3)
    loss = loss.cpu().numpy().astype(np.float64)
    _, grad = hip.easgd_distill(gpu(z[None]), gpu(idx), gpu(val), teacher_lse=gpu(lse), labels=gpu(label), hard=0.3)
    assert np.abs((loss[:V] - loss[V:]) / (2 * step) - grad.cpu().numpy()[0]).max() < 1e-4


def test_repeats_are_the_same_bits_and_the_entries_agree():
    import paper_1708_02983_amd as hip
    rng = np.random.default_rng(4)
    gpu = lambda a: torch.from_numpy(a).cuda()
    for rows, V in ((600, 777), (64, 40000), (3, 200000)):
        z = torch.randn(rows, V, device="cuda").to(torch.bfloat16)
        idx, val, lse = teacher(rng, rows, V, 30, 1.0, twice=True)
        args = (z, gpu(idx), gpu(val))
        kw = dict(teacher_lse=gpu(lse), labels=gpu(rng.integers(-1, V, rows).astype(np.int32)), hard=0.5)
        a = hip.easgd_distill(*args, scale=64.0, **kw)
        loss, state = hip.easgd_distill_loss(*args, **kw)
        grad = hip.easgd_distill_grad(*args, state, scale=64.0, **kw)
        assert torch.equal(loss, a[0]) and torch.equal(grad, a[1])
        for _ in range(3):
            b = hip.easgd_distill(*args, scale=64.0, **kw)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_rows():
    import paper_1708_02983_amd as hip
    z = torch.randn(0, 30, device="cuda")
    loss, grad = hip.easgd_distill(z, torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda"))
    assert loss.shape == (0,) and grad.shape == (0, 30)
