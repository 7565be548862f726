"""Oracle of the operators around the MoDSE layer: float64 numpy written from their formulas, no rounding in between.
Test infrastructure only; shares no code with the HIP path."""
from __future__ import annotations

from typing import Optional

import numpy as np

E4M3_MAX = 448.0


def norm_fwd(x, residual, gamma, eps):
    """h = x + residual, y = gamma h / sqrt(mean(h^2) + eps), rstd."""
    h = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h, h * rstd[:, None] * np.asarray(gamma, np.float64), rstd


def scales(y, group):
    """max|y| / 448 of every row (group 0) or of every `group` columns of it."""
    t, d = y.shape
    width = group or d
    n = -(-d // width)
    padded = np.zeros((t, n * width))
    padded[:, :d] = np.abs(y)
    s = np.maximum(padded.reshape(t, n, width).max(2) / E4M3_MAX, 2.0 ** -126)
    return s, np.repeat(s, width, axis=1)[:, :d]


def e4m3_values(codes):
    """The values of bytes in e4m3: sign, 4 exponent bits of bias 7, 3 fraction bits; S.1111.111 is NaN, no infinity."""
    c = np.asarray(codes).astype(np.int64)
    sign, e, f = np.where(c & 128, -1.0, 1.0), c >> 3 & 15, c & 7
    v = np.where(e == 0, f / 8.0 * 2.0 ** -6, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    return np.where(c & 127 == 127, np.nan, sign * v)


def norm_bwd(h, gamma, rstd, dY, dH=None):
    """dX, dgamma of <dY, y> + <dH, h> for the stored h."""
    h, gamma, dY = (np.asarray(a, np.float64) for a in (h, gamma, dY))
    r = np.asarray(rstd, np.float64)[:, None]
    hat, g = h * r, dY * gamma
    dX = r * (g - hat * (g * hat).mean(1, keepdims=True))
    if dH is not None:
        dX = dX + np.asarray(dH, np.float64)
    return dX, (dY * hat).sum(0)


def log_softmax(logits):
    """log p (NaN nowhere: -inf for masked entries and for all of a row that has no others), and which rows have entries."""
    x = np.asarray(logits, np.float64)
    m = x.max(1)
    some = m > -np.inf
    z = x - np.where(some, m, 0.0)[:, None]
    with np.errstate(divide="ignore"):
        return z - np.where(some, np.log(np.exp(z).sum(1)), 0.0)[:, None], some


def logprobs_fwd(logits, targets=None, top=0):
    """logp, entropy, top_idx, top_logp."""
    lp, some = log_softmax(logits)
    t, v = lp.shape
    logp = None
    if targets is not None:
        targets = np.asarray(targets, np.int64)
        logp = np.where(targets < 0, 0.0, lp[np.arange(t), np.clip(targets, 0, v - 1)])
        logp = np.where(targets >= v, np.nan, logp)
    p = np.exp(lp)
    entropy = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(1)
    idx = np.argsort(-np.asarray(logits, np.float64), axis=1, kind="stable")[:, :top]
    idx = np.concatenate([idx, np.zeros((t, top - idx.shape[1]), idx.dtype)], 1)
    value = np.take_along_axis(lp, idx, 1)
    value[:, v:] = -np.inf
    return logp, entropy, np.where(value == -np.inf, -1, idx), value


def logprobs_bwd(logits, targets, d_logp, d_entropy: Optional[np.ndarray] = None):
    """Gradient of sum d_logp logp + d_entropy entropy."""
    lp, some = log_softmax(logits)
    t, v = lp.shape
    p = np.exp(lp)
    g = np.zeros((t, v))
    if targets is not None:
        targets = np.asarray(targets, np.int64)
        has = (targets >= 0) & some
        w = np.where(has, np.asarray(d_logp, np.float64), 0.0)
        g -= w[:, None] * p
        g[np.arange(t), np.clip(targets, 0, v - 1)] += w
        g[(targets >= v) & some] = np.nan
    if d_entropy is not None:
        plogp = np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0)
        g -= np.where(some, np.asarray(d_entropy, np.float64), 0.0)[:, None] * (plogp - p * plogp.sum(1, keepdims=True))
    return g


def orthogonalize(G, coeffs, eps):
    """X = G / (|G| + eps), then X <- a X + (b A + c A^2) X with A = X X^T for every (a, b, c)."""
    X = np.asarray(G, np.float64)
    X = X / (np.sqrt((X * X).sum()) + eps)
    for a, b, c in coeffs:
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
    return X
