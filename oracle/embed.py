"""Embedding lookups and the gradient of their table in float64."""
from __future__ import annotations

import numpy as np


def embed_forward(table, tokens, scale=1.0):
    """scale table[tokens]; a token outside [0, V) gives zeros."""
    table, tokens = np.asarray(table, np.float64), np.asarray(tokens)
    x = np.zeros(tokens.shape + table.shape[1:])
    held = (tokens >= 0) & (tokens < table.shape[0])
    x[held] = scale * table[tokens[held]]
    return x


def embed_backward(tokens, dx, V, scale=1.0, old=None):
    """old (or zeros [V, D]) + scale * the sums of dx over equal tokens."""
    dx = np.asarray(dx, np.float64)
    d = np.zeros((V, dx.shape[-1])) if old is None else np.asarray(old, np.float64).copy()
    for t, row in zip(np.asarray(tokens).ravel(), dx.reshape(-1, dx.shape[-1])):
        if 0 <= t < V:
            d[t] += scale * row
    return d
