"""The AdamW step in float64, and the 8-bit states' code: rows of 256 with one scale."""
from __future__ import annotations

import numpy as np

ROW = 256


def adamw(p, g, m, v, lr, beta1, beta2, eps, step, weight_decay, grad_scale=1.0):
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    up = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - lr * (weight_decay * p + up), m, v


def _rows(n):
    return np.arange(n) // ROW


def dequant(cm, cv, m_scale, v_scale):
    r = _rows(len(cm))
    cm = cm.astype(np.float64) / 127
    return np.sign(cm) * cm * cm * np.asarray(m_scale, np.float64)[r], \
        (cv.astype(np.float64) / 255) ** 4 * np.asarray(v_scale, np.float64)[r]


def neighbours(x, scale, power, top):
    """The two codes next to |x| (float64) in its row and the chance of the upper one."""
    s = np.asarray(scale, np.float64)[_rows(len(x))]
    w = np.where(s > 0, np.abs(x) / np.where(s > 0, s, 1.0), 0.0)
    lo = np.minimum(np.floor(w ** (1 / power) * top), top - 1)
    a, b = (lo / top) ** power, ((lo + 1) / top) ** power
    return lo, (w - a) / (b - a)


def row_max(x):
    return np.maximum.reduceat(np.abs(x), np.arange(0, len(x), ROW))
