"""Oracle of the calls on given tokens: log probabilities, entropy, rank, alternatives, their gradient and the loss made of them.

Plain numpy in 64 bits, one row after the other, written from the definitions in ``include/easgd.h``.
"""
from __future__ import annotations

import numpy as np

from .logits import log_softmax, order


def _given(token, V):
    return token is not None and 0 <= token < V


def score(z, token=None, temperature=1.0, k=0):
    """logprob, entropy, rank of one row and its k first alternatives (log probabilities, places); token None: the row has none."""
    z = np.asarray(z, np.float64)
    V = len(z)
    top, places = np.full(k, -np.inf), np.full(k, -1, np.int64)
    if token is not None and not 0 <= token < V:
        return 0.0, 0.0, -1, top, places
    first = order(z)
    rank = 0
    if token is not None:
        rank = int(np.flatnonzero(first == token)[0]) if z[token] > -np.inf else len(first)
    places[:min(k, len(first))] = first[:k]
    if not (z > -np.inf).any() and not np.isnan(z).any():
        return -np.inf if token is not None else 0.0, 0.0, rank, top, places
    with np.errstate(invalid="ignore", divide="ignore"):
        log_q = log_softmax(z, temperature)
        q = np.exp(log_q)
        entropy = -np.where(q == 0.0, 0.0, q * np.where(np.isneginf(log_q), 0.0, log_q)).sum()
    if not np.isfinite(z.max()):
        log_q = np.full(V, np.nan)
        entropy = np.nan
    top[:min(k, len(first))] = log_q[first[:k]]
    return (log_q[token] if token is not None else 0.0), entropy, rank, top, places


def score_grad(z, token, temperature=1.0, dlogprob=0.0, dentropy=0.0):
    """The gradient of dlogprob * logprob + dentropy * entropy of one row."""
    z = np.asarray(z, np.float64)
    V = len(z)
    if token is not None and not 0 <= token < V:
        return np.zeros(V)
    if not (z > -np.inf).any() and not np.isnan(z).any():
        return np.zeros(V)
    if not np.isfinite(z.max()):
        return np.full(V, np.nan)
    log_q = log_softmax(z, temperature)
    q = np.exp(log_q)
    log_q = np.where(q > 0.0, log_q, 0.0)
    entropy = -(q * log_q).sum()
    d = -dlogprob * q - dentropy * q * (log_q + entropy)
    if token is not None:
        d[token] += dlogprob
    return d / temperature


def token_loss(z, token, weight=1.0, bonus=0.0, temperature=1.0):
    """-weight * logprob - bonus * entropy of one row, and its gradient."""
    z = np.asarray(z, np.float64)
    if not 0 <= token < len(z) or (not (z > -np.inf).any() and not np.isnan(z).any()):
        return 0.0, np.zeros(len(z))
    logprob, entropy, *_ = score(z, token, temperature)
    loss = (-weight * logprob if weight != 0.0 else 0.0) - (bonus * entropy if bonus != 0.0 else 0.0)
    if np.isnan(entropy):
        loss = np.nan
    return loss, score_grad(z, token, temperature, -weight, -bonus)
