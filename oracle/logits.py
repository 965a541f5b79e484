"""Oracle of the calls on rows of logits: top logits, distillation from a teacher's top logits, sampling.

Plain numpy in 64 bits, one row after the other, written from the definitions in ``include/easgd.h``.
"""
from __future__ import annotations

import numpy as np


def order(z):
    """Indices of the logits above -inf, larger logits first, equal ones by ascending index (NaN counts as masked)."""
    z = np.asarray(z, np.float64)
    there = np.flatnonzero(z > -np.inf)
    return there[np.lexsort((there, -z[there]))]


def logsumexp(z, T=1.0):
    """Differences are taken before they are divided: quotients of large logits would round away what they differ by."""
    z = np.asarray(z, np.float64)
    m = z.max() if z.size else -np.inf
    if not np.isfinite(m):
        return m
    return m / T + np.log(np.exp((z - m) / T).sum())


def log_softmax(z, T=1.0):
    """The maximum is taken off first: logits near the ends of a type's range would absorb the logarithm of the sum."""
    z = np.asarray(z, np.float64)
    t = (z - z.max()) / T
    return t - np.log(np.exp(t).sum())


def top_logits(z, k, temperature=1.0):
    """values [k], indices [k] (-inf and -1 where nothing is left), log-sum-exp at the temperature."""
    z = np.asarray(z, np.float64)
    first = order(z)[:k]
    values, indices = np.full(k, -np.inf), np.full(k, -1, np.int64)
    values[:len(first)], indices[:len(first)] = z[first], first
    lse = np.inf if (z == np.inf).any() else np.nan if np.isnan(z).any() else logsumexp(z, temperature)
    return values, indices, lse


def _teacher(V, indices, values, teacher_lse, T):
    """Probability of every slot (0 for slots that are not used) and the target of every place."""
    indices = np.asarray(indices)
    used = (indices >= 0) & (indices < V)
    a = np.where(used, np.where(used, values, 0.0).astype(np.float64) / T, -np.inf)
    live = a != -np.inf                  # the others have probability 0, whatever the log-sum-exp is
    if teacher_lse == -np.inf:
        live[:] = False                  # the teacher's row is masked
    log_p = np.full(len(a), -np.inf)
    if live.any():
        log_p[live] = a[live] - teacher_lse if teacher_lse is not None else log_softmax(a[live])
    p = np.where(used, np.exp(log_p), 0.0)
    target = np.zeros(V)
    np.add.at(target, indices[used], p[used])
    return used, p, log_p, target


def distill(z, indices, values, teacher_lse=None, label=None, temperature=1.0, hard=0.0):
    """loss and d loss / d z of one row; label None: no labels were given."""
    z = np.asarray(z, np.float64)
    V, T = len(z), float(temperature)
    zero = 0.0, np.zeros(V)
    if label is not None and not 0 <= label < V:
        return zero
    if not (z > -np.inf).any() and not np.isnan(z).any():
        return zero
    used, p, log_p, target = _teacher(V, indices, values, teacher_lse, T)
    log_q = log_softmax(z, T)
    q = np.exp(log_q)
    places = np.unique(np.asarray(indices)[used])
    outside = np.ones(V, bool)
    outside[places] = False
    log_R = logsumexp(log_q[outside])        # R itself may be too small for 64 bits
    r = max(0.0, 1.0 - p.sum()) if teacher_lse is not None else 0.0
    if log_R == -np.inf:
        r = 0.0
    kl = 0.0
    for i in np.flatnonzero(p > 0):
        kl += p[i] * (log_p[i] - log_q[indices[i]])
    if r > 0.0:
        kl += r * (np.log(r) - log_R)
    c = p.sum() + r
    soft = c * q - target
    if r > 0.0:
        soft[outside] -= r * np.exp(log_softmax(z[outside], T))      # every place's share of R
    loss, grad = 0.0, np.zeros(V)
    if hard < 1.0:
        loss += (1.0 - hard) * T * T * kl
        grad += (1.0 - hard) * T * soft
    if hard > 0.0:
        log_q = log_softmax(z)
        loss -= hard * log_q[label]
        onehot = np.zeros(V)
        onehot[label] = 1.0
        grad += hard * (np.exp(log_q) - onehot)
    return loss, grad


def sample_token(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """token (-1: every logit is masked), log of its probability among the tokens that may be drawn, and how far u times their
    mass is from the nearest border between two tokens, relative to the mass."""
    z = np.asarray(z, np.float64)
    seq = order(z)
    if len(seq) == 0:
        return -1, np.nan, np.inf
    if not temperature > 0.0:
        return int(seq[0]), 0.0, np.inf
    best = z[seq[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(z[seq] == best, 1.0, 0.0 if best == np.inf else np.exp((z[seq] - best) / temperature))
    n = len(seq)
    if top_k >= 1:
        n = min(n, int(top_k))
    n_p = n_m = n
    if top_p < 1.0:
        run, need = 0.0, top_p * w[:n].sum()
        for n_p in range(1, n + 1):
            run += w[n_p - 1]
            if run >= need:
                break
    if min_p > 0.0:
        n_m = max(1, int((w >= min_p).sum()))
    n = min(n, n_p, n_m)
    kept = np.sort(seq[:n])
    weight = dict(zip(seq[:n].tolist(), w[:n].tolist()))
    mass = sum(weight[j] for j in kept.tolist())
    u = min(max(float(u), 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    run, gap, token = 0.0, np.inf, -1
    for j in kept.tolist():
        run += weight[j]
        if j != kept[-1]:
            gap = min(gap, abs(run - u * mass) / mass)
        if token < 0 and run > u * mass:
            token = j
    return token, float(np.log(weight[token] / mass)), gap
