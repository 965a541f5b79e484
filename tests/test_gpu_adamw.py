"""adamw_round with moments in 32 and 8 bits and easgd_grad_norms against the oracle: the moments bit for bit, the parameters to rounding."""
import numpy as np
import pytest
import torch

from oracle import adamw as oa

pytestmark = pytest.mark.gpu
F = np.float32
U = 2.0 ** -24
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def hip():
    import paper_1708_02983_amd as pkg
    return pkg


def padded(x, ld, fill=float("nan")):
    """[P][N] as [P][ld] on the GPU, with NaN behind the rows: a read there shows, and so does a write."""
    out = torch.full((x.shape[0], ld), fill, dtype=torch.float32, device="cuda")
    out[:, :x.shape[1]] = torch.from_numpy(x)
    return out


def problem(P, N, ld, dtype, seed, center, tensors, clip):
    rng = np.random.default_rng(seed)
    W = (rng.normal(size=(P, N)) * 0.1).astype(F)
    size = np.exp(rng.normal(size=N) * 2) * 1e-3
    G = torch.from_numpy((rng.normal(size=(P, N)) * size).astype(F)).to(DTYPES[dtype])
    M = (rng.normal(size=(P, N)) * size * 0.3).astype(F)
    S = ((rng.normal(size=(P, N)) * size) ** 2 * 0.5).astype(F)
    Wc = (W.mean(axis=0) + rng.normal(size=N) * 0.01).astype(F) if center else None
    table = None
    if tensors:
        ends = np.sort(rng.integers(0, N + 1, tensors))
        if tensors > 2:
            ends[1] = ends[0]                           # an empty tensor
        if tensors % 2:
            ends[-1] = N
        table = (ends, rng.uniform(0.5, 1.5, tensors).astype(F), rng.uniform(0, 0.1, tensors).astype(F))
    c = None
    if clip:
        c = rng.uniform(0.1, 1.0, P).astype(F)
        c[P // 2] = 0.0
        if P > 1:
            G[P // 2] = float("nan")
    return W, M, S, G, Wc, table, c


def device_tensors(table):
    if table is None:
        return None
    return tuple(torch.from_numpy(np.ascontiguousarray(t)).cuda() for t in (table[0].astype(np.int64), table[1], table[2]))


RULE = dict(eta=3e-3, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.02)


def check_parameters(dW, dWc, want, want_c, size, W, Wc, alpha):
    """A parameter is rounded once at the end; what it moves by is a dozen roundings of its terms, whose magnitudes `size` adds up (the exponents of
    sqrt and of the quotient among them).  A center is rounded once, its sum P times."""
    N, P = W.shape[1], W.shape[0]
    got = dW[:, :N].double().cpu().numpy()
    assert (np.abs(got - want) <= U * (np.abs(want) + 16 * size) + 1e-45).all(), np.abs(got - want).max()
    assert torch.isnan(dW[:, N:]).all()
    if Wc is not None:
        apart = np.abs(W.astype(np.float64)).sum(axis=0) + P * np.abs(Wc)
        got = dWc.double().cpu().numpy()
        assert (np.abs(got - want_c) <= U * (np.abs(want_c) + (P + 4) * alpha * apart)).all()


SHAPES = [(1, 1), (1, 3), (2, 5), (3, 255), (4, 256), (1, 257), (5, 1000), (16, 7850), (33, 2049), (2, 100003), (1, 1 << 20), (8, 300001)]


@pytest.mark.parametrize("P,N", SHAPES)
@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("eight", [False, True])
def test_rounds(hip, P, N, center, eight):
    for case, (dtype, extra, tensors, clip) in enumerate((("fp32", -N % 4, 0, False), ("bf16", 3, 5, True), ("fp16", -N % 4 + 4, 2, True), ("fp32", 1, 300, False))):
        ld, seed, step = N + extra, 1000 * P + N + case, 1 + 7 * case
        W, M, S, G, Wc, table, clip = problem(P, N, ld, dtype, seed, center, tensors, clip)
        rho = 0.3 if center else 0.0
        dW, dWc = padded(W, ld), None if Wc is None else torch.from_numpy(Wc).cuda()
        dG = torch.full((P, ld), float("nan"), dtype=DTYPES[dtype], device="cuda")
        dG[:, :N] = G
        kw = dict(Wc=dWc, rho=rho, tensors=device_tensors(table), clip=None if clip is None else torch.from_numpy(clip).cuda(), N=N, **RULE)
        G64 = G.float().numpy()
        if eight:
            codes = [oa.encode(M[i], S[i], i, 0, 5) for i in range(P)]
            mc, vc, ms, vs = (np.stack(t) for t in zip(*codes))
            M, S = oa.decode_m(mc, ms), oa.decode_s(vc, vs)
            dM, dS = (torch.full((P, ld), 0x55, dtype=torch.uint8, device="cuda") for _ in range(2))
            dM[:, :N], dS[:, :N] = torch.from_numpy(mc), torch.from_numpy(vc)
            dms, dvs = torch.from_numpy(ms).cuda(), torch.from_numpy(vs).cuda()
            hip.adamw_round(dW, dM.view(torch.float8_e4m3fn), dS.view(torch.float8_e5m2), dG, step, M_scale=dms, S_scale=dvs, seed=seed, **kw)
        else:
            dM, dS = padded(M, ld), padded(S, ld)
            hip.adamw_round(dW, dM, dS, dG, step, **kw)
        torch.cuda.synchronize()
        want, want_c, M1, S1, size = oa.adamw_round(W, M, S, G64, Wc, step, RULE["eta"], rho, RULE["beta1"], RULE["beta2"], RULE["eps"], RULE["decay"], table, clip)
        check_parameters(dW, dWc, want, want_c, size, W, Wc, RULE["eta"] * rho)
        if not eight:
            for d, x in ((dM, M1), (dS, S1)):
                assert np.array_equal(d[:, :N].cpu().numpy(), x) and torch.isnan(d[:, N:]).all()
            continue
        for i in range(P):
            new = oa.encode(M1[i], S1[i], i, step, seed) if clip is None or clip[i] != 0.0 else (mc[i], vc[i], ms[i], vs[i])
            for d, x in zip((dM, dS, dms, dvs), new):
                assert np.array_equal(d[i, :len(x)].cpu().numpy(), x), (i, case)
        assert (dM[:, N:] == 0x55).all() and (dS[:, N:] == 0x55).all()


@pytest.mark.parametrize("power", [-140, -100, -64, -20, 20, 60])
@pytest.mark.parametrize("eight", [False, True])
def test_sizes_of_numbers(hip, power, eight):
    """Gradients from subnormal numbers up to where squares leave 32 bits: moments, codes and scales bit for bit."""
    P, N, ld = 2, 700, 700
    W, M, S, G, *_ = problem(P, N, ld, "fp32", power + 200, False, 0, False)
    M, S = np.zeros_like(M), np.zeros_like(S)
    G = (G.numpy().astype(np.float64) * 2.0 ** power).astype(F)
    G[0, :256:3] = 0.0
    dW = padded(W, ld)
    kw = dict(RULE, eps=1e-30)
    if eight:
        dM, dS = torch.zeros((P, ld), dtype=torch.uint8, device="cuda"), torch.zeros((P, ld), dtype=torch.uint8, device="cuda")
        ms, vs = torch.zeros((P, 3), device="cuda"), torch.zeros((P, 3), device="cuda")
    else:
        dM, dS = padded(M, ld), padded(S, ld)
    for step in (1, 2):
        if eight:
            hip.adamw_round(dW, dM.view(torch.float8_e4m3fn), dS.view(torch.float8_e5m2), torch.from_numpy(G).cuda(), step, M_scale=ms, S_scale=vs, seed=4, **kw)
        else:
            hip.adamw_round(dW, dM, dS, torch.from_numpy(G).cuda(), step, **kw)
        want, _, M, S, size = oa.adamw_round(W, M, S, G, None, step, kw["eta"], 0.0, kw["beta1"], kw["beta2"], kw["eps"], kw["decay"])
        # (terms below 2^-126 in products are subnormal: 2^-149 each; a root of a subnormal square has the square's own error and is left out)
        fine = (S == 0.0) | (S > 2.0 ** -100)
        off = np.abs(dW.double().cpu().numpy() - want) - U * (np.abs(want) + 16 * size)
        assert (off[fine] <= 0).all() and torch.isfinite(dW).all()
        W = dW.cpu().numpy()
        if not eight:
            assert np.array_equal(dM.cpu().numpy(), M) and np.array_equal(dS.cpu().numpy(), S)
            continue
        for i in range(P):
            new = oa.encode(M[i], S[i], i, step, 4)
            for d, x in zip((dM, dS, ms, vs), new):
                assert np.array_equal(d[i].cpu().numpy(), x), (i, step)
        M, S = oa.decode_m(dM.cpu().numpy(), ms.cpu().numpy()), oa.decode_s(dS.cpu().numpy(), vs.cpu().numpy())


@pytest.mark.parametrize("eight", [False, True])
def test_step_and_rate_in_memory(hip, eight):
    P, N, ld = 3, 1000, 1000
    W, M, S, G, Wc, table, clip = problem(P, N, ld, "fp32", 3, True, 4, True)
    results = []
    for in_memory in (False, True):
        dW, dWc, dG = padded(W, ld), torch.from_numpy(Wc).cuda(), G.cuda()
        kw = dict(Wc=dWc, rho=0.2, tensors=device_tensors(table), clip=torch.from_numpy(clip).cuda(), beta1=0.9, beta2=0.99)
        if eight:
            dM, dS = torch.zeros((P, ld), dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros((P, ld), dtype=torch.float8_e5m2, device="cuda")
            kw.update(M_scale=torch.zeros((P, 4), device="cuda"), S_scale=torch.zeros((P, 4), device="cuda"), seed=8)
        else:
            dM, dS = torch.zeros((P, ld), device="cuda"), torch.zeros((P, ld), device="cuda")
        for t in (1, 2, 3, 5000000000):
            step, eta = (torch.tensor([t], device="cuda"), torch.tensor([0.01 / t], device="cuda")) if in_memory else (t, float(F(0.01 / t)))
            hip.adamw_round(dW, dM, dS, dG, step, eta, **kw)
        results.append([t.clone().view(torch.uint8) for t in (dW, dM, dS, dWc)])
    for x, y in zip(*results):
        assert torch.equal(x, y)


def test_moments_that_are_not_finite(hip):
    P, N = 1, 600
    for bad in (float("inf"), float("nan")):
        dW, dG = torch.ones((P, N), device="cuda"), torch.full((P, N), 1e-3, device="cuda")
        dG[0, 300] = bad
        dM, dS = torch.zeros((P, N), dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros((P, N), dtype=torch.float8_e5m2, device="cuda")
        ms, vs = torch.zeros((P, 3), device="cuda"), torch.zeros((P, 3), device="cuda")
        hip.adamw_round(dW, dM, dS, dG, 1, 0.1, M_scale=ms, S_scale=vs)
        assert torch.isnan(dW).sum() == 1 and torch.isnan(dW[0, 300])
        assert torch.isnan(ms[0]).tolist() == [False, True, False] and torch.isnan(vs[0]).tolist() == [False, True, False]


@pytest.mark.parametrize("P,N", [(1, 1), (3, 7), (2, 255), (5, 8192), (4, 8193), (16, 100003), (200, 300), (1, 5000001)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_norms(hip, P, N, dtype):
    rng = np.random.default_rng(N)
    ld = N + rng.integers(0, 5)
    G = torch.full((P, ld), float("nan"), device="cuda")
    G[:, :N] = torch.from_numpy((rng.normal(size=(P, N)) * 10.0 ** rng.uniform(-4, 2, (P, 1))).astype(F))
    G = G.to(DTYPES[dtype])
    if P > 2:
        G[1, N // 2] = float("inf")
        G[2, N - 1] = float("nan")
    norm, clip = hip.easgd_grad_norms(G, max_norm=2.0, N=N)
    want, want_clip = oa.norms(G[:, :N].double().cpu().numpy(), 2.0)
    # squares and sums in 64 bits: one rounding to 32, and 2^-53 a term
    for got, x in ((norm, want), (clip, want_clip)):
        got = got.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(x))
        fine = np.isfinite(x)
        assert (np.abs(got - x)[fine] <= (U + 2.0 ** -50) * np.abs(x)[fine]).all() and np.array_equal(got[~fine & ~np.isnan(x)], x[~fine & ~np.isnan(x)])
    again = hip.easgd_grad_norms(G, max_norm=2.0, N=N)
    assert torch.equal(norm.view(torch.int32), again[0].view(torch.int32))


def test_norms_at_the_ends_of_the_type(hip):
    G = torch.tensor([[1e30, 1e30], [1e-40, 0.0], [0.0, 0.0], [3e38, 3e38]], device="cuda")
    norm, clip = hip.easgd_grad_norms(G, max_norm=1.0)
    want = np.sqrt((G.double().cpu().numpy() ** 2).sum(axis=1))
    assert np.allclose(norm[:2].double().cpu().numpy(), want[:2], rtol=2 * U, atol=1e-45) and norm[2] == 0.0 and norm[3] == float("inf")
    assert np.allclose(clip.double().cpu().numpy(), [1 / want[0], 1.0, 1.0, 0.0], rtol=2 * U)
    assert hip.easgd_grad_norms(G)[1].tolist() == [1.0, 1.0, 1.0, 0.0]
