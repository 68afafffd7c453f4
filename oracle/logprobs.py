"""Log probabilities, entropy and likeliest tokens of one row of logits, from the definitions in 64 bits."""
import numpy as np


def row(x, temperature, token, top):
    """(log probability of token, entropy, the likeliest tokens, their log probabilities)"""
    x = x.astype(np.float64) / (temperature if np.isfinite(temperature) and temperature > 0 else 1.0)
    live = ~np.isneginf(x)
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))[:top] if not np.isnan(x).any() else None
    if not live.any():
        return -np.inf, 0.0, order, np.full(top, -np.inf)
    m = x[live].max()
    with np.errstate(invalid="ignore"):
        norm = m + np.log(np.exp(x[live] - m).sum())
        logp = x - norm
        entropy = -(np.exp(logp[live]) * logp[live]).sum()
    return (logp[token] if 0 <= token < len(x) else -np.inf), entropy, order, None if order is None else logp[order]
