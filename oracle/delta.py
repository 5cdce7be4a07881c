"""The gated delta rule, token by token in float64: forward and gradient.

    S' = e^g S;  e = v - S'^T k;  u = beta e;  S = S' + k u^T;  y = scale S^T q
"""
from __future__ import annotations

import numpy as np


def delta_forward(q, k, v, g, beta, seq_len=None, S0=None, scale=None):
    """q, k [T,B,Hk,Dk], v [T,B,Hv,Dv], g, beta [T,B,Hv]: (y, ST, tape)."""
    q, k, v, g, beta = (np.asarray(a, np.float64) for a in (q, k, v, g, beta))
    T, B, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    scale = 1.0 / np.sqrt(Dk) if scale is None else scale
    seq_len = np.full(B, T) if seq_len is None else seq_len
    S = np.zeros((B, Hv, Dk, Dv)) if S0 is None else np.asarray(S0, np.float64).copy()
    y = np.zeros((T, B, Hv, Dv))
    states, errs = [], []
    for t in range(T):
        states.append(S.copy())
        err = np.zeros((B, Hv, Dv))
        S = S.copy()
        for b in range(B):
            if t >= seq_len[b]:
                continue
            for h in range(Hv):
                hk = h // (Hv // Hk)
                Sd = np.exp(g[t, b, h]) * S[b, h]
                err[b, h] = v[t, b, h] - Sd.T @ k[t, b, hk]
                S[b, h] = Sd + np.outer(k[t, b, hk], beta[t, b, h] * err[b, h])
                y[t, b, h] = scale * (S[b, h].T @ q[t, b, hk])
        errs.append(err)
    tape = dict(q=q, k=k, v=v, g=g, beta=beta, seq_len=seq_len, scale=scale, states=states + [S], errs=errs)
    return y, S, tape


def delta_backward(tape, dy, dST=None):
    """Gradients dict(dq, dk, dv, dg, dbeta, dS0)."""
    q, k, v, g, beta = (tape[n] for n in ("q", "k", "v", "g", "beta"))
    T, B, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    dS = np.zeros((B, Hv, Dk, Dv)) if dST is None else np.asarray(dST, np.float64).copy()
    out = {n: np.zeros(a.shape) for n, a in (("dq", q), ("dk", k), ("dv", v), ("dg", g), ("dbeta", beta))}
    for t in reversed(range(T)):
        for b in range(B):
            if t >= tape["seq_len"][b]:
                continue
            for h in range(Hv):
                hk = h // (Hv // Hk)
                d = np.asarray(dy[t, b, h], np.float64)
                S, e = tape["states"][t + 1][b, h], tape["errs"][t][b, h]
                kt, qt, bt, a = k[t, b, hk], q[t, b, hk], beta[t, b, h], np.exp(g[t, b, h])
                out["dq"][t, b, hk] += tape["scale"] * (S @ d)
                D = dS[b, h] + tape["scale"] * np.outer(qt, d)
                du = D.T @ kt
                out["dbeta"][t, b, h] = du @ e
                de = bt * du
                out["dv"][t, b, h] = de
                Sd = a * tape["states"][t][b, h]
                out["dk"][t, b, hk] += D @ (bt * e) - Sd @ de
                D = D - np.outer(kt, de)
                out["dg"][t, b, h] = (D * Sd).sum()
                dS[b, h] = a * D
    out["dS0"] = dS
    return out
