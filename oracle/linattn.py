"""Linear attention with a decay for each head, token by token in float64: forward
and gradient.

    S = e^g S + k v^T;  y = scale S^T q
"""
from __future__ import annotations

import numpy as np


def linattn_forward(q, k, v, g, seq_len=None, S0=None, scale=None):
    """q, k [T,B,Hk,Dk], v [T,B,Hv,Dv], g [Hv]: (y, ST, tape)."""
    q, k, v, g = (np.asarray(a, np.float64) for a in (q, k, v, g))
    T, B, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    scale = 1.0 / np.sqrt(Dk) if scale is None else scale
    seq_len = np.full(B, T) if seq_len is None else seq_len
    S = np.zeros((B, Hv, Dk, Dv)) if S0 is None else np.asarray(S0, np.float64).copy()
    y = np.zeros((T, B, Hv, Dv))
    states = []
    for t in range(T):
        S = S.copy()
        for b in range(B):
            if t >= seq_len[b]:
                continue
            for h in range(Hv):
                hk = h // (Hv // Hk)
                S[b, h] = np.exp(g[h]) * S[b, h] + np.outer(k[t, b, hk], v[t, b, h])
                y[t, b, h] = scale * (S[b, h].T @ q[t, b, hk])
        states.append(S)
    return y, S, dict(q=q, k=k, v=v, g=g, seq_len=seq_len, scale=scale, states=states)


def linattn_backward(tape, dy, dST=None):
    """Gradients dict(dq, dk, dv, dS0)."""
    q, k, v, g = (tape[n] for n in ("q", "k", "v", "g"))
    T, B, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    dS = np.zeros((B, Hv, Dk, Dv)) if dST is None else np.asarray(dST, np.float64).copy()
    out = {n: np.zeros(a.shape) for n, a in (("dq", q), ("dk", k), ("dv", v))}
    for t in reversed(range(T)):
        for b in range(B):
            if t >= tape["seq_len"][b]:
                continue
            for h in range(Hv):
                hk = h // (Hv // Hk)
                d = np.asarray(dy[t, b, h], np.float64)
                out["dq"][t, b, hk] += tape["scale"] * (tape["states"][t][b, h] @ d)
                D = dS[b, h] + tape["scale"] * np.outer(q[t, b, hk], d)
                out["dk"][t, b, hk] += D @ v[t, b, h]
                out["dv"][t, b, h] = D.T @ k[t, b, hk]
                dS[b, h] = np.exp(g[h]) * D
    out["dS0"] = dS
    return out
