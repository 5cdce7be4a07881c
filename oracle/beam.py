"""One step of beam search, candidate by candidate in float64."""
from __future__ import annotations

import numpy as np


def beam_select(logits, scores, finished=None, lengths=None, eos=-1, length_penalty=0.0):
    """logits [B*K, V], the others [B, K]: dict of parents, tokens, scores, finished,
    lengths [B, K] and the rank of each search's candidates in order (for telling how near
    the last one is to the next)."""
    logits, scores = np.asarray(logits, np.float64), np.asarray(scores, np.float64)
    B, K = scores.shape
    V = logits.shape[1]
    finished = np.zeros((B, K), int) if finished is None else np.asarray(finished)
    lengths = np.zeros((B, K), int) if lengths is None else np.asarray(lengths)
    out = dict(parents=np.tile(np.arange(K), (B, 1)), tokens=np.full((B, K), -1), scores=np.full((B, K), -np.inf),
               finished=np.zeros((B, K), int), lengths=lengths.copy())
    ranks = []
    for b in range(B):
        score = np.full((K, V), -np.inf)
        length = np.zeros((K, V), int)
        for k in range(K):
            if not scores[b, k] > -np.inf:
                continue
            if finished[b, k]:
                score[k, max(eos, 0)], length[k] = scores[b, k], max(0, lengths[b, k])
                continue
            x = logits[b * K + k]
            m = x.max()
            if not np.isfinite(m):           # nothing allowed, or no number
                continue
            score[k] = scores[b, k] + ((x - m) - np.log(np.exp(x - m).sum()))
            length[k] = max(0, lengths[b, k]) + 1
        rank = (score / ((5.0 + length) / 6.0) ** length_penalty).ravel()
        order = np.argsort(-rank, kind="stable")
        order = order[rank[order] > -np.inf]
        ranks.append(rank[order])
        for place, at in enumerate(order[:K]):
            k, t = divmod(int(at), V)
            done = bool(finished[b, k])
            out["parents"][b, place] = k
            out["tokens"][b, place] = eos if done else t
            out["scores"][b, place] = score[k, t]
            out["finished"][b, place] = done or t == eos
            out["lengths"][b, place] = length[k, t]
    return dict(out, ranks=ranks)


def beam_slots(parents, slots):
    """The slots of the next beams and the copies (from, to) that they need: a beam's
    first successor keeps its slot, further ones get those of beams without any.  -1: no
    state, which all its successors have, and no place for one."""
    parents, slots = np.asarray(parents), np.asarray(slots)
    out, copies = np.full_like(slots, -1), []
    for b in range(len(parents)):
        seen = set()
        free = [k for k in range(parents.shape[1]) if k not in parents[b] and slots[b, k] != -1]
        for k, p in enumerate(parents[b]):
            if p not in seen:
                out[b, k] = slots[b, p]
            elif slots[b, p] >= 0 and free:
                out[b, k] = slots[b, free.pop(0)]
                copies.append((int(slots[b, p]), int(out[b, k])))
            seen.add(p)
    return out, copies
