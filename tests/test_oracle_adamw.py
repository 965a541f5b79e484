"""The oracle of the AdamW rounds against torch's optimizer, hand values, and what random rounding promises."""
import numpy as np
import torch

from oracle import adamw as oa

F = np.float32
rng = np.random.default_rng(9)


def test_against_torchs_optimizer():
    N = 50
    w0 = rng.normal(size=N)
    p = torch.tensor(w0, dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([p], lr=0.02, betas=(0.75, 0.9375), eps=2.0 ** -10, weight_decay=0.125)
    W, M, S = w0.astype(F)[None], np.zeros((1, N), F), np.zeros((1, N), F)
    for t in range(1, 6):
        g = rng.normal(size=N).astype(F)
        p.grad = torch.tensor(g.astype(np.float64))
        opt.step()
        W, _, M, S, _ = oa.adamw_round(W.astype(F), M, S, g[None], None, t, 0.02, beta1=0.75, beta2=0.9375, eps=2.0 ** -10, decay=0.125)
    assert np.allclose(W[0], p.detach().numpy(), rtol=0, atol=2e-6)


def test_exchange_and_clip():
    W, Wc = np.array([[1.0], [3.0]], F), np.array([1.0], F)
    zero = np.zeros((2, 1), F)
    got, c, M, S, _ = oa.adamw_round(W, zero, zero, zero, Wc, 1, 0.5, rho=0.5, decay=0.0)
    assert got.tolist() == [[1.0], [2.5]] and c.tolist() == [1.5]
    G = np.full((2, 1), np.nan, F)
    got, _, M, S, _ = oa.adamw_round(W, zero, zero, G, None, 1, 0.5, clip=[0.0, 0.0])
    assert (got == W).all() and not M.any() and not S.any()
    norm, clip = oa.norms(np.array([[3.0, 4.0], [0.3, 0.4], [np.inf, 1.0], [np.nan, 1.0], [0.0, 0.0]]), 1.0)
    assert np.allclose(norm[:2], [5.0, 0.5]) and clip[0] == 0.2 and clip[1:].tolist() == [1.0, 0.0, 0.0, 1.0]


def test_tensors():
    rate, dec = oa.per_parameter(6, ([2, 2, 5], [0.5, 9.0, 0.25], [0.0, 9.0, 0.125]), 0.5)
    assert rate.tolist() == [0.5, 0.5, 0.25, 0.25, 0.25, 1.0] and dec.tolist() == [0, 0, 0.125, 0.125, 0.125, 0.5]


def test_codes_are_the_types_own():
    """Every code stands for what torch's types of 8 bits say."""
    code = torch.arange(256, dtype=torch.uint8)
    one = np.ones((1, 1), F)
    for dtype, decode in ((torch.float8_e4m3fn, oa.decode_m), (torch.float8_e5m2, oa.decode_s)):
        with np.errstate(invalid="ignore"):
            assert np.array_equal(decode(code.numpy()[None], one)[0], code.view(dtype).float().numpy(), equal_nan=True)


def test_rounding_is_to_a_neighbour_and_exact_on_average():
    N = 256
    m = (rng.normal(size=N) * np.exp(rng.normal(size=N) * 3)).astype(F)
    v = (m * m * F(0.3)).astype(F)
    steps = 400
    sum_m, sum_v = np.zeros(N), np.zeros(N)
    for t in range(steps):
        mc, vc, ms, vs = oa.encode(m, v, 3, t, 77)
        dm, dv = oa.decode_m(mc[None], ms[None])[0], oa.decode_s(vc[None], vs[None])[0]
        gap_m, gap_v = np.maximum(np.abs(m) / 8, 2.0 ** -9 * ms[0]), np.maximum(v / 4, 2.0 ** -16 * vs[0])
        assert (np.abs(dm - m) <= gap_m).all() and (np.abs(dv - v) <= gap_v).all() and ((dv > 0) == (v > 0)).all()
        sum_m += dm
        sum_v += dv
    # the mean of `steps` roundings, each off by at most one gap with standard deviation of at most half of it: five deviations, and 2^-17 of a gap
    # for the 16 bits; the smallest of v are never rounded to 0, which moves them up
    assert (np.abs(sum_m / steps - m) <= gap_m * (2.5 / np.sqrt(steps) + 2.0 ** -17)).all()
    # log v has a standard deviation of 6.4 and its largest of 256 is some 2.8 of them up: 2^-31 below that is about 0.6 down, 3 of 4 are above
    high = v > 2.0 ** -16 * vs[0]
    assert high.sum() > 128 and (np.abs(sum_v / steps - v) <= gap_v * (2.5 / np.sqrt(steps) + 2.0 ** -17))[high].all()


def test_random_bits():
    """Each of the 65536 values about as often as any other, and neighbours, workers, steps and seeds that have nothing in common."""
    j = np.arange(1 << 18)
    r = oa.dither(j, 0, 1, 0) / 65536.0
    assert abs(r.mean() - 0.5) < 5 / np.sqrt(12 * len(j)) + 2.0 ** -17
    for other in (oa.dither(j, 1, 1, 0), oa.dither(j, 0, 2, 0), oa.dither(j, 0, 1, 1), np.roll(oa.dither(j, 0, 1, 0), 1), np.roll(oa.dither(j, 0, 1, 0), 2),
                  np.roll(oa.dither(j, 0, 1, 0), 4)):
        assert abs(np.corrcoef(r, other / 65536.0)[0, 1]) < 5 / np.sqrt(len(j))
    count = np.bincount((r * 256).astype(int), minlength=256)
    assert (np.abs(count - 1024) < 6 * 32).all()


def test_blocks_with_nothing_or_without_end():
    zero = np.zeros(300, F)
    mc, vc, ms, vs = oa.encode(zero, zero, 0, 1, 0)
    assert not mc.any() and not vc.any() and np.isfinite(ms).all()
    m = zero.copy()
    m[260] = np.inf
    mc, vc, ms, vs = oa.encode(m, zero, 0, 1, 0)
    assert np.isfinite(ms[0]) and np.isnan(ms[1]) and np.isfinite(vs).all()
    tiny = np.full(3, 1e-44, F)
    mc, vc, ms, vs = oa.encode(tiny, tiny, 0, 1, 0)
    assert (vc >= 1).all()


def test_the_smallest_second_moments_are_held_where_they_cannot_fall_below():
    """What is exact on average and what is not: an S below 2^-16 of its block's scale is always stored as that, whatever the random bits are, and stays there
    as it decays; from there on up the mean is S itself."""
    largest = F(1.5 * 2.0 ** 14)                        # the block's scale is 1
    S = np.array([largest, 2.0 ** -16 * 0.999, 2.0 ** -40, 2.0 ** -149, 0.0, 2.0 ** -16, 2.0 ** -16 * 1.25], F)
    seen = []
    for step in range(1, 400):
        _, codes, _, scale = oa.encode(np.zeros_like(S), S, 0, step, 3)
        assert scale[0] == 1.0 and codes[1:6].tolist() == [1, 1, 1, 0, 1]
        seen.append(oa.decode_s(codes[None], scale[None])[0])
    assert set(seen[i][6] for i in range(len(seen))) == {F(2.0 ** -16), F(2.0 ** -15)}
    # 399 roundings with a deviation of less than half a step each: five deviations
    assert abs(np.mean([x[6] for x in seen]) - S[6]) < 2.0 ** -16 * 2.5 / np.sqrt(len(seen))
