"""Oracle of the AdamW rounds and of the norms that clip gradients.

The moments' arithmetic is pinned (every operation in 32 bits rounded on its own) and so are the codes of moments held in 8 bits: numpy in
32 bits gives the same bits.  What the parameters move by is computed in 64 bits.
"""
from __future__ import annotations

import numpy as np

F = np.float32
BLOCK = 256


def norms(G, max_norm):
    """norm and clip of every worker's gradient."""
    G = np.asarray(G, np.float64)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        norm = np.sqrt((G * G).sum(axis=1))
        clip = np.where(norm <= max_norm, 1.0, max_norm / norm)
        return norm, np.where(np.isfinite(norm.astype(F)), clip, 0.0)


def mix(x):
    x = np.atleast_1d(np.asarray(x, np.uint64)) & np.uint64(0xFFFFFFFF)
    x = (x ^ (x >> np.uint64(16))) * np.uint64(0x6C8E9CF5) & np.uint64(0xFFFFFFFF)
    x = (x ^ (x >> np.uint64(15))) * np.uint64(0x2F5D7A4B) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def dither(j, worker, step, seed):
    """16 random bits of parameters j of a worker in a step."""
    j = np.asarray(j, np.uint64)
    word = (j >> np.uint64(1)) & np.uint64(1)
    key = mix(int(mix((seed + worker * 0x9E3779B1) & 0xFFFFFFFF)[0]) + (step & 0xFFFFFFFF) * 0x85157AF5 % (1 << 32) + (word * np.uint64(0x632BE5AB)))
    h = mix((j >> np.uint64(2)) ^ key)
    return (h >> (np.uint64(16) * (j & np.uint64(1)))) & np.uint64(0xFFFF)


def _value(code, bits):
    """What a code of an 8-bit floating point type with `bits` of fraction stands for (without its sign)."""
    code = np.asarray(code, np.int64) & 0x7F
    e, f = code >> bits, code & ((1 << bits) - 1)
    bias = 7 if bits == 3 else 15
    value = np.where(e == 0, f / 2.0 ** bits * 2.0 ** (1 - bias), (1.0 + f / 2.0 ** bits) * 2.0 ** (e - bias).astype(np.float64))
    if bits == 3:
        return np.where(code == 0x7F, np.nan, value)
    return np.where(e == 31, np.where(f == 0, np.inf, np.nan), value)


def decode_m(code, scale):
    """[P][N] codes and [P][blocks] scales as fp32 numbers."""
    code = np.asarray(code)
    sign = np.where(code & 0x80, F(-1), F(1))
    return (sign * _value(code, 3).astype(F)) * np.repeat(np.asarray(scale, F), BLOCK, axis=1)[:, :code.shape[1]]


def decode_s(code, scale):
    code = np.asarray(code)
    sign = np.where(code & 0x80, F(-1), F(1))
    return (sign * _value(code, 2).astype(F)) * np.repeat(np.asarray(scale, F), BLOCK, axis=1)[:, :code.shape[1]]


def _encode(x, bits, top, r):
    """Codes and scale of one block of magnitudes, r: 16 random bits each.  From the definition: neighbours and their distances."""
    if not np.isfinite(x).all():
        return np.zeros(len(x), np.uint8), F(np.nan)
    most = float(x.max())
    e = max(int(np.frexp(most)[1]) - 1 - top, -126) if most > 0 else -126
    bias = 7 if bits == 3 else 15
    y = (x * F(2.0 ** -e) * F(2.0 ** (bias - 127))).view(np.uint32).astype(np.int64)     # the type's exponents are those of fp32
    low, rest = y >> (23 - bits), y & ((1 << (23 - bits)) - 1)
    up = rest + r.astype(np.int64) * (1 << (7 - bits)) + (1 << (6 - bits)) >= 1 << (23 - bits)
    return (low + up).astype(np.uint8), F(2.0 ** e)


def encode(m, v, worker, step, seed):
    """Codes and scales of one worker's new moments."""
    N = len(m)
    blocks = (N + BLOCK - 1) // BLOCK
    mc, vc = np.zeros(N, np.uint8), np.zeros(N, np.uint8)
    ms, vs = np.zeros(blocks, F), np.zeros(blocks, F)
    r = dither(np.arange(N), worker, step, seed)
    for b in range(blocks):
        at = slice(b * BLOCK, min((b + 1) * BLOCK, N))
        code, ms[b] = _encode(np.abs(m[at]), 3, 7, r[at])
        mc[at] = code | np.signbit(m[at]).astype(np.uint8) << 7
        code, vs[b] = _encode(v[at], 2, 14, r[at])
        vc[at] = np.maximum(code, (v[at] > 0) & np.isfinite(vs[b]))
    return mc, vc, ms, vs


def moments(m, v, g, beta1, beta2):
    """New moments: every operation in 32 bits rounded on its own."""
    b1, b2 = F(beta1), F(beta2)
    with np.errstate(over="ignore", invalid="ignore"):
        return m * b1 + g * (F(1) - b1), v * b2 + (g * (F(1) - b2)) * g


def per_parameter(N, tensors, decay):
    """rate and decay of every parameter."""
    rate, dec = np.ones(N), np.full(N, float(F(decay)))
    if tensors is not None:
        begin = 0
        for end, r, d in zip(*tensors):
            rate[begin:end], dec[begin:end] = r, d
            begin = max(begin, int(end))
    return rate, dec


def adamw_round(W, M, S, G, Wc, step, eta, rho=0.0, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.01, tensors=None, clip=None):
    """The round on [P][N] fp32 arrays (G any type).  Returns W, Wc in 64 bits, M, S in 32, and per parameter of W the sum of the
    magnitudes of what it was moved by (for error bounds)."""
    P, N = W.shape
    eta, rho, eps = float(F(eta)), float(F(rho)), float(F(eps))
    b1, b2 = float(F(beta1)), float(F(beta2))
    by1, by2 = 1.0 / (1.0 - b1 ** step), 1.0 / (1.0 - b2 ** step)
    rate, dec = per_parameter(N, tensors, decay)
    W64, M, S = W.astype(np.float64), M.copy(), S.copy()
    moved = np.zeros((P, N))
    size = np.zeros((P, N))
    for i in range(P):
        c = F(1) if clip is None else F(clip[i])
        if c == 0:
            continue
        g = c * np.asarray(G[i], F)
        rough = np.abs(M[i]).astype(np.float64) * b1 + np.abs(g).astype(np.float64) * (1 - b1)
        M[i], S[i] = moments(M[i], S[i], g, beta1, beta2)
        with np.errstate(invalid="ignore", over="ignore"):
            d = np.sqrt(S[i].astype(np.float64) * by2) + eps
            moved[i] = eta * rate * (M[i].astype(np.float64) * by1 / d + dec * W64[i])
            size[i] = np.abs(eta) * rate * (rough * by1 / d + np.abs(dec * W64[i]))
    if Wc is None:
        return W64 - moved, None, M, S, size
    apart = W64 - Wc.astype(np.float64)
    size += np.abs(eta * rho) * (np.abs(W64) + np.abs(Wc))
    return W64 - moved - eta * rho * apart, Wc + eta * rho * apart.sum(axis=0), M, S, size
