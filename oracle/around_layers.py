"""Plain definitions of the calls around the layers: norms, steps of AdamW with their 8-bit states, adapters.

numpy only; shares no code with the kernels.  Everything is float64 but the step of AdamW, which is defined operation by operation in
float32, so that codes that are rounded by chance come out the same.
"""
from __future__ import annotations

import math

import numpy as np

F32 = np.float32


# ------------------------------------------------------------------ norm
def rms_norm(h, gain, eps):
    """(y, rstd) of rows h."""
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)
    return h * rstd[:, None] * gain[None, :], rstd


def rms_norm_gradient(dy, h, gain, rstd, dh):
    """(dx, dgain) with rstd as it is given."""
    n, w = h * rstd[:, None], dy * gain[None, :]
    dx = (w - n * np.mean(w * n, axis=1, keepdims=True)) * rstd[:, None]
    return dx + (0.0 if dh is None else dh), (dy * n).sum(axis=0)


# ------------------------------------------------------------------ 8-bit states
def mix(x):
    x ^= x >> 16
    x = (x * 0x85A308D3) & 0xFFFFFFFF
    x ^= x >> 15
    x = (x * 0x9E3779B1) & 0xFFFFFFFF
    return x ^ (x >> 16)


def chance(seed, step, place):
    """32 random bits of one element."""
    key = mix(((seed & 0xFFFFFFFF) + mix(((seed >> 32) + mix(step & 0xFFFFFFFF)) & 0xFFFFFFFF)) & 0xFFFFFFFF)
    return mix(((place & 0xFFFFFFFF) + mix(((place >> 32) + key) & 0xFFFFFFFF)) & 0xFFFFFFFF)


def state_values(bits):
    """The magnitudes that the codes of one sign stand for, before the group's scale; bits: of the significand."""
    out = []
    for c in range(16 << bits):
        e, s = c >> bits, c & ((1 << bits) - 1)
        out.append(s * 2.0 ** (-14 - bits) if e == 0 else (1 + s / 2.0 ** bits) * 2.0 ** (e - 15))
    return np.array(out)


def state_restore(codes, scales, is_signed):
    bits = 3 if is_signed else 4
    c = codes.astype(int)
    v = state_values(bits)[c & 127 if is_signed else c]
    if is_signed:
        v = np.where(c & 128, -v, v)
    f = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return v * np.repeat(f, 32)


def state_save(x, chances, is_signed):
    """(codes, scale bytes) of float32 numbers, groups filled with zeros: to the code below or above, as the rest and the chance (of 65536) add up."""
    bits = 3 if is_signed else 4
    levels = state_values(bits)
    n = -(-len(x) // 32)
    codes, scales = np.zeros(32 * n, dtype=np.uint8), np.zeros(n, dtype=np.uint8)
    for g in range(n):
        v = x[32 * g:32 * g + 32]
        if not np.all(np.isfinite(v)):
            scales[g] = 255
            continue
        big = float(np.max(np.abs(v)))
        f = math.frexp(big)[1] - 1
        f = min(max(f + int(math.ldexp(big, -f) > levels[-1]), -100), 120) if big > 0 else -100
        scales[g] = f + 127
        for i, one in enumerate(v):
            y = math.ldexp(abs(float(one)), -f)
            low = min(int(np.searchsorted(levels, y, side="right")) - 1, len(levels) - 1)
            step = 2.0 ** (max(low >> bits, 1) - 15 - bits)
            # (of the rest as many bits count as a float's significand has)
            rest = math.floor((y - levels[low]) / step * 2 ** (23 - bits))
            c = low + ((rest + (int(chances[32 * g + i]) << (7 - bits))) >> (23 - bits))
            c = min(c, len(levels) - 1)
            if not is_signed and one > 0:
                c = max(c, 1)
            codes[32 * g + i] = c | (128 if is_signed and np.signbit(one) else 0)
    return codes, scales


def power(b, n):
    r = 1.0
    while n:
        if n & 1:
            r *= b
        n >>= 1
        b *= b
    return r


def adamw(p, g, m, v, lr, step, beta1, beta2, eps, decay, scale):
    """One step in float32, operation by operation; v is the second moment.  Returns (p, m, v, sqrt(v), what p changed by beside its decay)."""
    g = g.astype(F32) * F32(scale)
    m = F32(beta1) * m + F32(1.0 - beta1) * g
    v = F32(beta2) * v + (F32(1.0 - beta2) * g) * g
    root = np.sqrt(v)
    by = (F32(lr / (1.0 - power(beta1, step))) * m) / (root * F32(1.0 / math.sqrt(1.0 - power(beta2, step))) + F32(eps))
    return p * F32(1.0 - lr * float(F32(decay))) - by, m, v, root, by


# ------------------------------------------------------------------ adapters
def adapters(X, ids, A, B, scale, base):
    """(Y, U), token by token."""
    T, r, F = X.shape[0], A.shape[1], B.shape[2]
    Y = np.zeros((T, F)) if base is None else base.copy()
    U = np.zeros((T, r))
    for t in range(T):
        i = int(ids[t])
        if 0 <= i < A.shape[0]:
            U[t] = A[i] @ X[t]
            Y[t] += scale[i] * (U[t] @ B[i])
    return Y, U


def adapters_gradient(dY, X, U, ids, A, B, scale, base):
    """(dX, dA, dB), token by token."""
    dX = np.zeros(X.shape) if base is None else base.copy()
    dA, dB = np.zeros(A.shape), np.zeros(B.shape)
    for t in range(X.shape[0]):
        i = int(ids[t])
        if 0 <= i < A.shape[0]:
            V = scale[i] * (B[i] @ dY[t])
            dX[t] += V @ A[i]
            dA[i] += np.outer(V, X[t])
            dB[i] += scale[i] * np.outer(U[t], dY[t])
    return dX, dA, dB
