"""Log probabilities of given tokens, entropy, alternatives and their gradient in float64."""
from __future__ import annotations

import numpy as np


def logprob_forward(x, targets=None, top_k=0):
    """x [N,V]: dict(lse, logp, entropy, p, lp, top_ids, top_logp).  A row of
    minus infinities has lse, logp, top_logp = -inf and entropy 0."""
    x = np.asarray(x, np.float64)
    N, V = x.shape
    m = x.max(1)
    empty = np.isneginf(m)
    e = np.exp(x - np.where(empty, 0.0, m)[:, None])
    s = e.sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(empty, -np.inf, m + np.log(np.where(empty, 1.0, s)))
    p = np.where(empty[:, None], 0.0, e / np.where(empty, 1.0, s)[:, None])
    # (x - m) - log s: their sum loses log s where m is as large as a type's lowest value
    lp = np.where(np.isneginf(x), -np.inf,
                  (x - np.where(empty, 0.0, m)[:, None]) - np.log(np.where(empty, 1.0, s))[:, None])
    plp = p * np.where(p > 0, lp, 0.0)
    out = dict(lse=lse, p=p, lp=lp, entropy=-plp.sum(1), empty=empty)
    if targets is not None:
        t = np.where((targets >= 0) & (targets < V), targets, -1)
        out["targets"] = t
        out["logp"] = np.where(t < 0, 0.0, lp[np.arange(N), np.maximum(t, 0)])
    if top_k:
        ids = np.argsort(-np.where(np.isnan(x), -np.inf, x), axis=1, kind="stable")[:, :top_k]
        out["top_ids"], out["top_logp"] = ids, np.take_along_axis(lp, ids, 1)
    return out


def logprob_backward(f, dlogp=None, dentropy=None, dtop=None):
    """dlogits of sum dlogp logp + dentropy entropy + sum dtop top_logp."""
    p, N = f["p"], len(f["p"])
    d = np.zeros_like(p)
    rows = np.arange(N)
    if dlogp is not None:
        w = np.where(f["targets"] < 0, 0.0, dlogp)
        d -= p * w[:, None]
        d[rows, np.maximum(f["targets"], 0)] += w
    if dentropy is not None:
        lp = np.where(p > 0, f["lp"], 0.0)
        d -= dentropy[:, None] * p * (lp + f["entropy"][:, None])
    if dtop is not None:
        d -= p * dtop.sum(1)[:, None]
        for j in range(dtop.shape[1]):
            np.add.at(d, (rows, f["top_ids"][:, j]), dtop[:, j])
    return np.where(f["empty"][:, None], 0.0, d)
