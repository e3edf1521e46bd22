"""Plain float64 definitions of the calls on a network's real-valued ends: saved inputs, 4-bit weights, the loss.

numpy only, one value or one token at a time where that is clearer; shares no code with the kernels.
"""
from __future__ import annotations

import math

import numpy as np

GROUP = 32
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _groups(row):
    return [row[i:i + GROUP] for i in range(0, len(row), GROUP)]


def group_exponent(values, top, too_large):
    """The exponent of a group: floor(log2 of the largest magnitude) - top, kept within -110 .. 120, one more where
    too_large(largest scaled magnitude); None if a value is not finite, -110 for zeros."""
    if not np.all(np.isfinite(values)):
        return None
    a = float(np.max(np.abs(values)))
    if a == 0.0:
        return -110
    e = min(max(math.frexp(a)[1] - 1 - top, -110), 120)
    return e + 1 if too_large(math.ldexp(a, -e)) else e


def round_half_even(x):
    return float(np.rint(x))


def save8(X):
    """X [rows, cols] -> (Q int8 [rows, 32 groups], S uint8 [rows, groups])."""
    rows, cols = X.shape
    n = -(-cols // GROUP)
    Q, S = np.zeros((rows, n * GROUP), dtype=np.int8), np.zeros((rows, n), dtype=np.uint8)
    for r in range(rows):
        for i, g in enumerate(_groups(X[r].astype(np.float64))):
            e = group_exponent(g, 6, lambda a: a >= 127.5)
            if e is None:
                S[r, i] = 255
                continue
            S[r, i] = e + 127
            Q[r, i * GROUP:i * GROUP + len(g)] = np.clip(np.rint(np.ldexp(g, -e)), -127, 127)
    return Q, S


def restore8(Q, S, cols):
    scale = np.where(S == 255, np.nan, np.ldexp(1.0, S.astype(int) - 127))
    return (Q.astype(np.float64) * np.repeat(scale, GROUP, axis=1))[:, :cols]


def code4(a):
    """Code of a scaled magnitude: the nearest level, the even code of two that are as near, 7 above."""
    best = min(range(8), key=lambda c: (abs(LEVELS[c] - a), c % 2))
    return best


def pack4(W):
    """W [F, K] -> (codes [F, 32 groups], exponents + 127 [F, groups]); 255 and codes 7 where a group is not finite."""
    F, K = W.shape
    n = -(-K // GROUP)
    codes, scale = np.zeros((F, n * GROUP), dtype=np.uint8), np.full((F, n), 17, dtype=np.uint8)
    for f in range(F):
        for i, g in enumerate(_groups(W[f].astype(np.float64))):
            e = group_exponent(g, 2, lambda a: a > 7.0)
            at = slice(i * GROUP, i * GROUP + len(g))
            if e is None:
                codes[f, i * GROUP:(i + 1) * GROUP], scale[f, i] = 7, 255
                continue
            scale[f, i] = e + 127
            codes[f, at] = [code4(a) for a in np.abs(np.ldexp(g, -e))]
            codes[f, at] |= (np.signbit(g).astype(np.uint8) << 3)
    return codes, scale


def value4(codes, scale, K):
    levels = np.array(LEVELS + tuple(-x for x in LEVELS))
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(int) - 127))
    return (levels[codes] * np.repeat(s, GROUP, axis=1))[:, :K]


def tiles4(codes, scale):
    """The layout of include/dab.h, element by element."""
    F, n = scale.shape
    Ft, Kt, K4 = -(-F // 16), -(-n // 4), -(-n // 16)
    Q, S = np.zeros((Ft, Kt, 64, 16), dtype=np.uint8), np.full((Ft, K4, 64, 4), 17, dtype=np.uint8)
    for f in range(F):
        for g in range(n):
            kt, lane = g // 4, (g % 4) * 16 + f % 16
            S[f // 16, kt // 4, lane, kt % 4] = scale[f, g]
            c = codes[f, g * GROUP:(g + 1) * GROUP]
            Q[f // 16, kt, lane] = c[0::2] | (c[1::2] << 4)
    return Q, S


def head(H, W, targets, g, ignore):
    """(loss, lse, P, dH, dW) of softmax cross entropy of H W^T, token by token."""
    T, V = H.shape[0], W.shape[0]
    H, W = H.astype(np.float64), W.astype(np.float64)
    loss, lse, P = np.zeros(T), np.zeros(T), np.zeros((T, V))
    live = np.zeros((T, 1), dtype=bool)
    for t in range(T):
        if targets[t] == ignore:
            continue
        if not 0 <= targets[t] < V:
            loss[t] = np.nan
            continue
        live[t] = True
        z = W @ H[t]
        m = np.max(z)
        lse[t] = m + math.log(np.sum(np.exp(z - m)))
        loss[t] = lse[t] - z[targets[t]]
        P[t] = np.exp(z - lse[t])
        P[t, targets[t]] -= 1.0
        P[t] *= g[t]
    return loss, lse, P, P @ W, P.T @ np.where(live, H, 0.0)
