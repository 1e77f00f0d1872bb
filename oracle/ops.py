"""Oracle of the language-model operators: dropout, token log-probabilities, the preference loss
and the clipped policy loss with a KL term, with their gradients.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Plain numpy in 64 bits, from the formulas;
shares nothing with the HIP library.  Inputs are arrays of any real type (taken to float64).
"""

import numpy as np

from . import rng

FIELD = 1 << 16


def keep_mask(p, seed, row_ids, cols):
    """bool[len(row_ids), cols]: value j of row r is kept when field j % 4 of output j // 4 of the
    stream seeded with output r of the stream `seed` reaches floor(65536 p + 1/2)."""
    threshold = int(np.floor(p * FIELD + 0.5))
    out = np.zeros((len(row_ids), cols), dtype=bool)
    for i, r in enumerate(row_ids):
        key = rng.splitmix64(seed, int(r) & rng.MASK64)
        for j in range(cols):
            out[i, j] = ((rng.splitmix64(key, j // 4) >> (16 * (j % 4))) & 0xFFFF) >= threshold
    return out


def keep_share(p):
    """Probability that a value is kept (p rounded to a multiple of 2^-16)."""
    return 1.0 - np.floor(p * FIELD + 0.5) / FIELD


def dropout(x, p, seed, row_ids, residual=None):
    x = np.asarray(x, dtype=np.float64)
    keep = keep_mask(p, seed, row_ids, x.shape[1])
    out = np.zeros_like(x)
    out[keep] = x[keep] / keep_share(p)
    return out if residual is None else out + np.asarray(residual, dtype=np.float64)


def row_stats(z):
    """(maximum, ln sum exp(z - maximum)) of each row; (-inf, 0) where a row holds nothing but -inf."""
    z = np.asarray(z, dtype=np.float64)
    top = np.empty(len(z))
    log_sum = np.empty(len(z))
    for t, row in enumerate(z):
        if np.isnan(row).any() or np.isposinf(row).any():
            top[t] = log_sum[t] = np.nan
        elif np.isneginf(row).all():
            top[t], log_sum[t] = -np.inf, 0.0
        else:
            top[t] = row.max()
            log_sum[t] = np.log(np.exp(row - top[t]).sum())
    return top, log_sum


def has_token(targets, cols):
    targets = np.asarray(targets, dtype=np.int64)
    return (targets >= 0) & (targets < cols)


def token_logprobs(z, targets):
    """Log-probabilities of the targets; 0 where there is no token."""
    z = np.asarray(z, dtype=np.float64)
    on = has_token(targets, z.shape[1])
    top, log_sum = row_stats(z)
    out = np.zeros(len(z))
    for t in np.flatnonzero(on):
        out[t] = -np.inf if np.isneginf(top[t]) else (z[t, targets[t]] - top[t]) - log_sum[t]
    return out


def token_logprobs_backward(z, targets, grad):
    """grad (onehot - softmax); 0 without a token, where grad is 0 and where nothing can occur."""
    z = np.asarray(z, dtype=np.float64)
    on = has_token(targets, z.shape[1])
    top, log_sum = row_stats(z)
    out = np.zeros_like(z)
    for t in np.flatnonzero(on):
        if grad[t] == 0 or np.isneginf(top[t]):
            continue
        with np.errstate(invalid="ignore"):
            out[t] = -float(grad[t]) * np.exp(z[t] - top[t] - log_sum[t])
            out[t, targets[t]] += float(grad[t])
    return out


def _sigmoid(h):
    return 1.0 / (1.0 + np.exp(-h)) if h >= 0 else np.exp(h) / (1.0 + np.exp(h))


def _softplus(h):
    return max(h, 0.0) + np.log1p(np.exp(-abs(h)))


def preference(z, targets, offsets, ref=None, beta=0.1, smoothing=0.0, scale=1.0, weights=None):
    """(loss, margins, logprobs, gradient of scale * sum(weights * loss) in the log-probabilities)."""
    z = np.asarray(z, dtype=np.float64)
    lp = token_logprobs(z, targets)
    on = has_token(targets, z.shape[1])
    each = np.where(on, lp - (0.0 if ref is None else np.asarray(ref, dtype=np.float64)), 0.0)
    pairs = (len(offsets) - 1) // 2
    loss, margins, grad = np.zeros(pairs), np.zeros(pairs), np.zeros(len(z))
    o = np.clip(offsets, 0, len(z))
    for i in range(pairs):
        won, lost = slice(o[2 * i], o[2 * i + 1]), slice(o[2 * i + 1], o[2 * i + 2])
        h = beta * (each[won].sum() - each[lost].sum())
        margins[i] = h
        # An infinite margin's loss is the limit: a term of weight 0 does not count.
        loss[i] = sum(weight * _softplus(x) for weight, x in ((1 - smoothing, -h), (smoothing, h)) if weight)
        w = 1.0 if weights is None else float(weights[i])
        if w == 0:
            continue
        g = scale * w * beta * (smoothing * _sigmoid(h) - (1 - smoothing) * _sigmoid(-h))
        grad[won], grad[lost] = g, -g
    return loss, margins, lp, grad


def policy(z, targets, old, advantages, ref=None, clip_low=0.2, clip_high=0.2, kl=0.0, scale=1.0, weights=None):
    """(loss, logprobs, gradient of scale * sum(weights * loss) in the log-probabilities)."""
    z = np.asarray(z, dtype=np.float64)
    lp = token_logprobs(z, targets)
    on = has_token(targets, z.shape[1])
    if weights is not None:
        on = on & (np.asarray(weights) != 0)
    loss, grad = np.zeros(len(z)), np.zeros(len(z))
    for t in np.flatnonzero(on):
        a, ratio = float(advantages[t]), np.exp(lp[t] - float(old[t]))
        slope = 0.0
        if a != 0:
            bound = min(max(ratio, 1 - clip_low), 1 + clip_high) * a
            loss[t] = -min(ratio * a, bound)
            slope = -ratio * a if ratio * a <= bound else 0.0
        if kl != 0:
            d = float(ref[t]) - lp[t]
            loss[t] += kl * (np.expm1(d) - d if d < np.inf else d)   # the limit, not inf - inf
            slope -= kl * np.expm1(d)
        grad[t] = scale * slope * (1.0 if weights is None else float(weights[t]))
    return loss, np.where(on, lp, 0.0), grad
