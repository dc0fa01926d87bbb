"""Plain CPU oracle of the operators around the masked linear layers: activation
checkpoints in 8 bits, layer norm and RMS norm with their backward passes, and the
masked linear's weight gradient.

TEST INFRASTRUCTURE ONLY, as roi_oracle: the slow statement of what the GPU library
computes, sharing no code with it.  float64 throughout; inputs are the exact values of
the tensors that the library is given.

The checkpoint's layout: blocks of 32 consecutive columns of a row share a power of two,
2^e, the least with max |x| <= 127.5 * 2^e (-126 <= e <= 121); codes are the nearest
integers to x / 2^e, ties to even, at most 127 in magnitude; scale byte e + 133.  A block
with an infinity or NaN has scale byte 255 and codes 0, and stands for NaN.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK, E_MIN, E_MAX, BIAS = 32, -126, 121, 133


def pitches(cols):
    """Codes and scale bytes of a row: whole blocks, and whole groups of four blocks."""
    return -(-cols // BLOCK) * BLOCK, -(-cols // (4 * BLOCK)) * 4


def exponent(a):
    """The least e in [E_MIN, E_MAX] with a <= 127.5 * 2^e (E_MAX where there is none)."""
    e = E_MIN
    if a > 0:
        # a = m 2^k, 1/2 <= m < 1; 127.5 = 0.99609375 * 2^7
        m, k = math.frexp(a)
        e = k - 7 if m <= 0.99609375 else k - 6
    return min(max(e, E_MIN), E_MAX)


def checkpoint_save(x):
    """x [rows, cols] float64 -> (codes int8, scales uint8), padding included."""
    rows, cols = x.shape
    pitch, spitch = pitches(cols)
    codes = np.zeros((rows, pitch), np.int8)
    scales = np.full((rows, spitch), E_MIN + BIAS, np.uint8)
    for r in range(rows):
        for b in range(0, cols, BLOCK):
            v = x[r, b:b + BLOCK]
            if not np.all(np.isfinite(v)):
                scales[r, b // BLOCK] = 255
                continue
            e = exponent(float(np.max(np.abs(v))))
            scales[r, b // BLOCK] = e + BIAS
            codes[r, b:b + len(v)] = np.clip(np.rint(np.ldexp(v, -e)), -127, 127)
    return codes, scales


def checkpoint_load(codes, scales, cols):
    """The values (float64) of a checkpoint's first `cols` columns."""
    s = np.repeat(scales.astype(np.int64), BLOCK, axis=1)[:, :cols]
    v = np.ldexp(codes[:, :cols].astype(np.float64), s - BIAS)
    return np.where(s == 255, np.nan, np.where(s < E_MIN + BIAS, 0.0, v))


def norm_fwd(x, kind, gamma, beta, eps):
    """(y, mean, rstd) of the rows of x; gamma and beta may be None (1 and 0)."""
    mean = x.mean(axis=1) if kind == "layer" else np.zeros(len(x))
    c = x - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(axis=1) + eps)
    y = c * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean, rstd


def norm_bwd(dy, x, kind, gamma, mean, rstd):
    """(dx, dgamma, dbeta) for the given statistics (mean ignored by the RMS norm)."""
    r = rstd[:, None]
    xh = (x - mean[:, None]) * r if kind == "layer" else x * r
    a = dy if gamma is None else dy * gamma
    dx = a - xh * (a * xh).mean(axis=1, keepdims=True)
    if kind == "layer":
        dx = dx - a.mean(axis=1, keepdims=True)
    return r * dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


def linear_wgrad(dY, x, acc=None):
    """sum_t dY[t, o] x[t, i] (+ acc)."""
    g = dY.T @ x
    return g if acc is None else g + acc
