"""Token log probabilities, entropy, most likely words and their gradient, in fp64 from the definitions.

TEST INFRASTRUCTURE ONLY.  Logits x [V, N], row = word, column = token.
"""
from __future__ import annotations

import numpy as np


def log_probs(x):
    """[V, N]; -infinity where the logit is (a column of nothing else: everywhere)."""
    x = np.asarray(x, dtype=np.float64)
    m = x.max(axis=0)
    with np.errstate(invalid="ignore", divide="ignore"):
        d = np.where(np.isneginf(m)[None], -np.inf, x - np.where(np.isneginf(m), 0.0, m))
        s = np.exp(d).sum(axis=0)
        return np.where(np.isneginf(m)[None], -np.inf, d - np.log(s))


def entropy(logp):
    with np.errstate(invalid="ignore"):
        p = np.exp(logp)
        return -np.where(p == 0, 0.0, p * logp).sum(axis=0)


def of_tokens(logp, tokens):
    tokens = np.asarray(tokens)
    V = logp.shape[0]
    at = logp[np.clip(tokens, 0, V - 1), np.arange(len(tokens))]
    return np.where(tokens < 0, 0.0, np.where(tokens >= V, np.nan, at))


def top(x, k):
    """Words [k, N] (-1 where there is none): by logit, equal ones by the lower word."""
    x = np.asarray(x, dtype=np.float64)
    out = np.full((k, x.shape[1]), -1, dtype=np.int64)
    for q in range(x.shape[1]):
        words = [v for v in range(x.shape[0]) if x[v, q] > -np.inf]
        words = sorted(words, key=lambda v: (-x[v, q], v))[:k]
        out[:len(words), q] = words
    return out


def grad(x, tokens, g_logp, g_entropy):
    """Gradient of sum(g_logp * log p of the tokens + g_entropy * entropy) with respect to x."""
    lp = log_probs(x)
    p = np.exp(lp)
    V, N = p.shape
    gl = np.zeros(N) if g_logp is None else np.where(np.asarray(tokens) < 0, 0.0, np.asarray(g_logp, dtype=np.float64))
    gh = np.zeros(N) if g_entropy is None else np.asarray(g_entropy, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        out = -gl * p - gh * np.where(p == 0, 0.0, p * (lp + entropy(lp)))
    if g_logp is not None:
        tokens = np.asarray(tokens)
        known = (tokens >= 0) & (tokens < V)
        out[tokens[known], np.arange(N)[known]] += gl[known]
        out[:, tokens >= V] = np.nan
    out[:, (gl == 0) & (gh == 0)] = 0.0
    return out
