"""Plain fp64 numpy definition of log probabilities, entropy and the most likely tokens of a logit row: test infrastructure only."""

import numpy as np


def row(z, token, temperature, top):
    """z [V] float64.  Returns (logprob, entropy, rank, top_tokens, top_logprobs)."""
    V = len(z)
    tokens, logprobs = np.full(top, -1), np.full(top, -np.inf)
    if np.isnan(z).any() or (z == np.inf).any():
        return np.nan, np.nan, -1, tokens, np.full(top, np.nan)
    known = 0 <= token < V
    rank = 1 + int((z > z[token]).sum() + (z[:token] == z[token]).sum()) if known else -1
    if (z == -np.inf).all():
        return -np.inf, 0.0, rank, tokens, logprobs
    y = z / temperature
    y = y - y.max()
    total = np.exp(y).sum()
    logp = y - np.log(total)
    p = np.exp(logp)
    entropy = -float((p[p > 0] * logp[p > 0]).sum())
    order = [v for v in np.lexsort((np.arange(V), -z))[:top] if z[v] > -np.inf]
    tokens[:len(order)], logprobs[:len(order)] = order, logp[order]
    return (logp[token] if known else -np.inf), entropy, rank, tokens, logprobs
