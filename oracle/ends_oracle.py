"""Oracle of the operators at both ends of a model: float64 numpy written from their formulas, no rounding in between.
Test infrastructure only; shares no code with the HIP path."""
from __future__ import annotations

import numpy as np


def embed_fwd(tokens, E, scale):
    tokens = np.asarray(tokens, np.int64)
    E = np.asarray(E, np.float64)
    x = scale * E[np.clip(tokens, 0, len(E) - 1)]
    x[tokens < 0] = 0.0
    x[tokens >= len(E)] = np.nan
    return x


def embed_bwd(tokens, dX, scale, vocab):
    """The gradient, the sum of the absolute values of its terms and their number."""
    tokens, dX = np.asarray(tokens, np.int64), np.asarray(dX, np.float64)
    dE, size, count = np.zeros((vocab, dX.shape[1])), np.zeros((vocab, dX.shape[1])), np.zeros(vocab, np.int64)
    for t, k in enumerate(tokens):
        if 0 <= k < vocab:
            dE[k] += scale * dX[t]
            size[k] += abs(scale) * np.abs(dX[t])
            count[k] += 1
    return dE, size, count


def head(x, W, targets, d_logp=None):
    """logp, log_z and, where d_logp is given, dX, dW and the gradient of the logits."""
    x, W, targets = np.asarray(x, np.float64), np.asarray(W, np.float64), np.asarray(targets, np.int64)
    t, v = len(x), len(W)
    logits = x @ W.T
    top = logits.max(1)
    log_z = top + np.log(np.exp(logits - top[:, None]).sum(1))
    rows = np.arange(t)
    logp = np.where(targets < 0, 0.0, logits[rows, np.clip(targets, 0, v - 1)] - log_z)
    logp[targets >= v] = np.nan
    if d_logp is None:
        return logp, log_z
    w = np.where(targets < 0, 0.0, np.asarray(d_logp, np.float64))
    G = -w[:, None] * np.exp(logits - log_z[:, None])
    G[rows, np.clip(targets, 0, v - 1)] += w
    G[targets >= v] = np.nan
    return logp, log_z, G @ W, G.T @ x, G


def philox4x32(counter, key, rounds):
    """The four words of Philox-4x32 (Salmon, Moraes, Dror and Shaw 2011) in Python's own integers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_bits(n, seed, offset, call):
    """16 random bits for each of n elements."""
    out = np.empty((n + 7) // 8 * 8, np.int64)
    for i in range(len(out) // 8):
        words = philox4x32((i, call, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32), 7)
        for w, word in enumerate(words):
            out[8 * i + 2 * w], out[8 * i + 2 * w + 1] = word & 0xFFFF, word >> 16
    return out[:n]


def dropout(x, residual, p, bits):
    limit = int(np.rint(p * 65536))
    x = np.asarray(x, np.float64)
    kept = bits.reshape(x.shape) >= limit
    with np.errstate(invalid="ignore"):
        y = np.where(kept, x * (65536 / (65536 - limit) if limit < 65536 else 0.0), 0.0)
    return y if residual is None else y + np.asarray(residual, np.float64), kept
