"""AdamW rounds of replicas that are long enough for tiles, the streaming forms of the kernels for short ones, and norms of gradients of which a block
reads several tiles: the moments bit for bit, the parameters to rounding."""
import numpy as np
import pytest
import torch

import test_gpu_adamw as base
from oracle import adamw as oa

pytestmark = pytest.mark.gpu
F = np.float32
U = 2.0 ** -24
RULE = base.RULE


@pytest.fixture(scope="module")
def hip():
    import paper_1708_02983_amd as pkg
    return pkg


@pytest.fixture
def streaming(hip):
    """Sets how the updates access memory (0: through the caches, 1: past them), and puts it back."""
    old = hip.get_option(hip.OPT_UPDATE_NONTEMPORAL)
    yield lambda how: hip.set_option(hip.OPT_UPDATE_NONTEMPORAL, how)
    hip.set_option(hip.OPT_UPDATE_NONTEMPORAL, old)


def least():
    """Parameters from which on every compute unit gets 64 blocks of 256, and tiles of several blocks are taken."""
    return 64 * 256 * torch.cuda.get_device_properties(0).multi_processor_count


def tensors_that_end_inside_blocks(rng, N):
    """Ends all over the replica, many of them within a few blocks, equal ones, and some among the last parameters."""
    ends = np.concatenate((rng.integers(0, N + 1, 300), 70000 + rng.integers(0, 300, 60), N - rng.integers(1, 600, 40), [70100, 70100]))
    ends = np.sort(ends)
    return ends, rng.uniform(0.5, 1.5, len(ends)).astype(F), rng.uniform(0, 0.1, len(ends)).astype(F)


def rows(x, ld, fill, dtype, skip=0):
    """[P][N] as [P][ld] on the GPU with `fill` behind the rows, `skip` elements behind an aligned address."""
    out = torch.full((skip + x.shape[0] * ld,), fill, dtype=dtype, device="cuda")[skip:].view(x.shape[0], ld)
    out[:, :x.shape[1]] = x if isinstance(x, torch.Tensor) else torch.from_numpy(x)
    return out


def check_parameters(dW, N, want, size):
    """As base.check_parameters, on the GPU: a parameter is rounded once at the end, what it moves by is a dozen roundings of its terms."""
    off = (dW[:, :N].double() - want).abs_() - U * (want.abs() + 16 * size) - 1e-45
    assert (off <= 0).all(), (off.argmax().item(), off.max().item())
    assert torch.isnan(dW[:, N:]).all()


@pytest.mark.parametrize("extra,dtype", [(0, "fp32"), (1, "bf16"), (255, "fp16"), (257, "fp32"), (5000, "bf16")])
def test_tiles_of_32_bits(hip, streaming, extra, dtype):
    P, N, step = 3, least() + extra, 1 + extra
    rng = np.random.default_rng(extra)
    W, M, S, G, Wc, _, clip = base.problem(P, N, N, dtype, extra + 7, True, 0, True)        # the second worker sits out, and its gradient is NaN
    table = tensors_that_end_inside_blocks(rng, N)
    G64, dt, kw = G.float().numpy(), base.DTYPES[dtype], dict(tensors=base.device_tensors(table), clip=torch.from_numpy(clip).cuda(), N=N, **RULE)
    for center in (False, True):
        c, rho = (Wc, 0.3) if center else (None, 0.0)
        want, want_c, M1, S1, size = oa.adamw_round(W, M, S, G64, c, step, RULE["eta"], rho, RULE["beta1"], RULE["beta2"], RULE["eps"], RULE["decay"], table, clip)
        want, size, M1, S1 = (torch.from_numpy(x).cuda() for x in (want, size, M1, S1))
        # rows at multiples of 16 bytes and at others, and all of them one element behind such an address
        for how, ld, skip in ((0, N + -N % 4, 0), (1, N + -N % 4 + 4, 0), (1, N + 1 + N % 2, 0), (0, N + 1 + N % 2, 0), (1, N + -N % 4 + 4, 1)):
            streaming(how)
            dW, dM, dS = (rows(x, ld, float("nan"), torch.float32, skip) for x in (W, M, S))
            dWc = None if c is None else rows(c[None], N, 0.0, torch.float32, skip)[0]
            hip.adamw_round(dW, dM, dS, rows(G, ld, float("nan"), dt, skip), step, Wc=dWc, rho=rho, **kw)
            check_parameters(dW, N, want, size)
            for d, x in ((dM, M1), (dS, S1)):
                assert torch.equal(d[:, :N], x) and torch.isnan(d[:, N:]).all(), (center, how, ld, skip)
            if center:
                alpha = RULE["eta"] * rho
                apart = np.abs(W.astype(np.float64)).sum(axis=0) + P * np.abs(Wc)
                assert (np.abs(dWc.double().cpu().numpy() - want_c) <= U * (np.abs(want_c) + (P + 4) * alpha * apart)).all()


@pytest.mark.parametrize("extra,dtype", [(0, "bf16"), (257, "fp32"), (5000, "fp16")])
def test_tiles_of_8_bits(hip, streaming, extra, dtype):
    P, N, step, seed = 3, least() + extra, 2 + extra, 1000 + extra
    blocks = (N + 255) // 256
    rng = np.random.default_rng(extra + 50)
    W, _, _, G, Wc, _, clip = base.problem(P, N, N, dtype, extra + 9, True, 0, True)
    table = tensors_that_end_inside_blocks(rng, N)
    # moments of about the gradients' size: codes of every kind under powers of two
    mc = (rng.integers(0, 0x78, (P, N)) | rng.integers(0, 2, (P, N)) << 7).astype(np.uint8)
    vc = rng.integers(0, 0x78, (P, N)).astype(np.uint8)
    ms, vs = (np.exp2(rng.integers(low, low + 6, (P, blocks))).astype(F) for low in (-20, -36))
    M, S = oa.decode_m(mc, ms), oa.decode_s(vc, vs)
    G64, dt = G.float().numpy(), base.DTYPES[dtype]
    dclip, dtable = torch.from_numpy(clip).cuda(), base.device_tensors(table)
    codes = None
    for center in (False, True):
        c, rho = (Wc, 0.3) if center else (None, 0.0)
        want, want_c, M1, S1, size = oa.adamw_round(W, M, S, G64, c, step, RULE["eta"], rho, RULE["beta1"], RULE["beta2"], RULE["eps"], RULE["decay"], table, clip)
        if codes is None:                               # the moments have nothing to do with the center
            new = [oa.encode(M1[i], S1[i], i, step, seed) if clip[i] != 0.0 else (mc[i], vc[i], ms[i], vs[i]) for i in range(P)]
            codes = [torch.from_numpy(np.stack(x)).cuda() for x in zip(*new)]
        want, size = torch.from_numpy(want).cuda(), torch.from_numpy(size).cuda()
        # rows of codes at multiples of 4 bytes (through the caches and past them), rows at others, and all of them one byte behind such an address
        for how, ld, skip in ((0, N + -N % 4, 0), (1, N + -N % 4 + 4, 0), (1, N + 1 + N % 2, 0), (0, N + -N % 4 + 4, 1)):
            streaming(how)
            dW = rows(W, ld, float("nan"), torch.float32)
            dM, dS = (rows(x, ld, 0x55, torch.uint8, skip) for x in (mc, vc))
            dms, dvs = torch.from_numpy(ms).cuda(), torch.from_numpy(vs).cuda()
            dWc = None if c is None else torch.from_numpy(c).cuda()
            hip.adamw_round(dW, dM.view(torch.float8_e4m3fn), dS.view(torch.float8_e5m2), rows(G, ld, float("nan"), dt), step, Wc=dWc, rho=rho, M_scale=dms, S_scale=dvs,
                            seed=seed, tensors=dtable, clip=dclip, N=N, **RULE)
            check_parameters(dW, N, want, size)
            for d, x in zip((dM[:, :N], dS[:, :N], dms, dvs), codes):
                assert torch.equal(d, x), (center, how, ld, skip)
            assert (dM[:, N:] == 0x55).all() and (dS[:, N:] == 0x55).all()
            if center:
                alpha = RULE["eta"] * rho
                apart = np.abs(W.astype(np.float64)).sum(axis=0) + P * np.abs(Wc)
                assert (np.abs(dWc.double().cpu().numpy() - want_c) <= U * (np.abs(want_c) + (P + 4) * alpha * apart)).all()


@pytest.mark.parametrize("P,N", [(1, 1), (3, 255), (4, 256), (5, 1000), (16, 7850), (33, 2049), (2, 100003)])
@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("eight", [False, True])
def test_short_replicas_past_the_caches(hip, streaming, P, N, center, eight):
    streaming(1)
    base.test_rounds(hip, P, N, center, eight)


@pytest.mark.parametrize("P,N", [(65535, 5), (40000, 300)])
@pytest.mark.parametrize("center", [False, True])
def test_many_workers(hip, P, N, center):
    W, M, S, G, Wc, table, clip = base.problem(P, N, N, "bf16", P, center, 3, True)
    rho = 0.3 if center else 0.0
    dW, dM, dS = (rows(x, N + 1, float("nan"), torch.float32) for x in (W, M, S))
    dWc = None if Wc is None else torch.from_numpy(Wc).cuda()
    hip.adamw_round(dW, dM, dS, rows(G, N + 1, float("nan"), torch.bfloat16), 4, Wc=dWc, rho=rho, tensors=base.device_tensors(table), clip=torch.from_numpy(clip).cuda(), N=N, **RULE)
    want, want_c, M1, S1, size = oa.adamw_round(W, M, S, G.float().numpy(), Wc, 4, RULE["eta"], rho, RULE["beta1"], RULE["beta2"], RULE["eps"], RULE["decay"], table, clip)
    base.check_parameters(dW, dWc, want, want_c, size, W, Wc, RULE["eta"] * rho)
    assert np.array_equal(dM[:, :N].cpu().numpy(), M1) and np.array_equal(dS[:, :N].cpu().numpy(), S1)


@pytest.mark.parametrize("P,N,dtype", [(16, 1863690, "fp32"), (3, 12000007, "fp32"), (5, 14000003, "bf16"), (1, 40000001, "fp16"), (3000, 40003, "fp32")])
def test_norms_of_several_tiles(hip, P, N, dtype):
    """From 64 MB on a block reads more than one tile.  Squares and sums in 64 bits on both sides: one rounding to 32, and sums of at most 2^12 terms one
    after the other, 2^-53 each."""
    gen = torch.Generator(device="cuda").manual_seed(N)
    ld = N + 3
    G = torch.full((P, ld), float("nan"), dtype=base.DTYPES[dtype], device="cuda")
    for row in G:
        row[:N] = torch.randn(N, generator=gen, device="cuda") * 1e-2
    norm, clip = hip.easgd_grad_norms(G, max_norm=0.5, N=N)
    want = torch.stack([row[:N].double().square().view(-1).sum().sqrt() for row in G])
    assert ((norm.double() - want).abs() <= (U + 2.0 ** -40) * want).all()
    assert ((clip.double() - (0.5 / want).clamp(max=1.0)).abs() <= (U + 2.0 ** -40) * (0.5 / want)).all()
