"""Many long rows, where every row is one block's: loss, gradient and top logits of sampled rows against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from logits_util import DTYPES, HALF_STEP, SMALLEST, sum_error
from oracle import logits as oracle
from test_gpu_distill import bounds, teacher

pytestmark = pytest.mark.gpu
F = np.float32


def matrix(rows, V, dtype, pad, offset, seed):
    """Random logits on the GPU, rows `pad` NaN apart and `offset` NaN behind the start of the buffer."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((offset + rows * (V + pad) + 16,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    z = buf[offset:offset + rows * (V + pad)].view(rows, V + pad)[:, :V]
    for at in range(0, rows, 64):
        z[at:at + 64] = torch.randn(min(64, rows - at), V, generator=gen, device="cuda") * 2
    return z


# rows that a block holds in registers with 12 slots a thread, that it reads again behind them, with 8 slots and 512 threads, again behind these, and
# a map of the teacher's places of more than 64 KB
@pytest.mark.parametrize("dtype, rows, V, pad", [
    ("bf16", 257, 17001, 0), ("fp16", 256, 24000, 8), ("bf16", 260, 50001, 3), ("fp16", 257, 50001, 0), ("bf16", 256, 65540, 0), ("fp16", 300, 70001, 1), ("bf16", 256, 131072, 0),
    ("bf16", 256, 530001, 7), ("bf16", 256, 1048576, 0), ("fp32", 257, 9001, 0), ("fp32", 256, 30001, 3), ("fp32", 256, 40001, 0), ("fp32", 256, 131072, 0)])
def test_loss_and_gradient(dtype, rows, V, pad):
    import paper_1708_02983_amd as hip
    z = matrix(rows, V, dtype, pad, pad % 4, V)
    sample = sorted({0, 1, 2, 3, rows // 2, rows - 2, rows - 1})
    rng = np.random.default_rng(V + rows)
    gpu = lambda a: None if a is None else torch.from_numpy(a).cuda()
    out = torch.empty_strided(z.shape, z.stride(), dtype=z.dtype, device="cuda")
    for n, (tail, T, hard) in enumerate(((False, 2.0, 0.5), (True, 1.0, 0.25), (True, 0.7, 0.4), (False, 0.7, 0.0), (True, 2.0, 0.3), (False, 1.5, 0.5))):
        T, hard = float(F(T)), float(F(hard))
        k = (64, 33, 256, 7, 130, 1)[n]
        idx, val, lse = teacher(rng, rows, V, k, T, twice=n % 2 == 0)
        labels = rng.integers(0, V, rows).astype(np.int32)
        labels[1], labels[rows - 2] = -1, V
        labels[3] = idx[3, 0] if 0 <= idx[3, 0] < V else labels[3]
        kw = dict(temperature=T, teacher_lse=gpu(lse) if tail else None, labels=gpu(labels) if hard else None, hard=hard)
        both_loss, both_grad = hip.easgd_distill(z, gpu(idx), gpu(val), scale=64.0, **kw)
        loss, state = hip.easgd_distill_loss(z, gpu(idx), gpu(val), **kw)
        dloss = rng.uniform(0.5, 2.0, rows).astype(F)
        grad = hip.easgd_distill_grad(z, gpu(idx), gpu(val), state, scale=64.0, dloss=gpu(dloss), dlogits=out, **kw)
        torch.cuda.synchronize()
        assert torch.equal(both_loss, loss)
        for r in sample:
            row = z[r].double().cpu().numpy()
            norm = np.float64(lse[r]) if tail else None
            label = int(labels[r]) if hard else None
            want, dz = oracle.distill(row, idx[r], val[r], norm, label, T, hard)
            if label is not None and not 0 <= label < V:
                assert loss[r] == 0 and not both_grad[r].any() and not grad[r].any()
                continue
            lt, gt = bounds(row, idx[r], val[r].astype(np.float64), norm, label, T, hard, 1.0, dtype)
            assert abs(loss[r].item() - want) <= lt + 2.0 ** -24 * abs(want), (n, r, loss[r].item(), want)
            for g, up in ((both_grad, 64.0), (grad, 64.0 * float(dloss[r]))):
                got, ref = g[r].double().cpu().numpy(), dz * up
                tol = gt * up + HALF_STEP[dtype] * (np.abs(ref) + gt * up) + 2.0 ** -24 * np.abs(ref) + SMALLEST[dtype] * (1 + up)
                bad = ~(np.abs(got - ref) <= tol)
                assert not bad.any(), (n, r, np.flatnonzero(bad)[:5], got[bad][:5], ref[bad][:5], tol[bad][:5])


@pytest.mark.parametrize("dtype, rows, V, k, pad", [
    ("bf16", 300, 20000, 64, 0), ("fp16", 256, 50001, 20, 0), ("fp32", 257, 40001, 33, 1), ("bf16", 256, 131072, 64, 0), ("fp32", 256, 20001, 256, 0), ("fp16", 256, 70001, 200, 3),
    ("bf16", 256, 20003, 1, 0)])
def test_top_logits(dtype, rows, V, k, pad):
    """Random rows, and among them rows that outgrow the list of candidates or keep raising its floor."""
    import paper_1708_02983_amd as hip
    z = matrix(rows, V, dtype, pad, pad, V + k)
    at = torch.arange(V, device="cuda")
    up = at * (40.0 / V) - 20.0
    special = {3: up, 4: -up, 5: torch.zeros(V, device="cuda"), 6: torch.where(at % 7 == 0, 2.0, 1.5), 7: (at % 5).float(), 8: up + torch.randn(V, device="cuda"),
               9: torch.where(at >= V - k, 60.0, -50.0), 10: torch.full((V,), float("-inf"), device="cuda"), 11: torch.where(at % (V // 40) == 1, 1.0 * (at % 11), float("-inf")),
               12: torch.where(at > V // 2, up, float("-inf")), 13: torch.where(at == V // 3, float("inf"), 0.0), 14: torch.where(at == V - 1, float("nan"), up)}
    for r, row in special.items():
        z[r] = row.to(z.dtype)
    T = 1.5
    values, indices, lse = hip.easgd_top_logits(z, k, temperature=T)
    again = hip.easgd_top_logits(z, k, temperature=T)
    torch.cuda.synchronize()
    assert all(torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) for x, y in zip((values, indices, lse), again))
    for r in [0, 1, 2, *special, rows // 2, rows - 1]:
        v, i, l = oracle.top_logits(z[r].double().cpu().numpy(), k, T)
        np.testing.assert_array_equal(indices[r].cpu().numpy(), i, err_msg=f"row {r}")
        np.testing.assert_array_equal(values[r].cpu().numpy(), v.astype(F), err_msg=f"row {r}")
        if np.isfinite(l):
            assert abs(lse[r].item() - l) <= sum_error(V) + 2.0 ** -24 * abs(l), (r, lse[r].item(), l)
        else:
            np.testing.assert_array_equal(lse[r].item(), l)
