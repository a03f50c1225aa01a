"""Activations, the gated product, 8-bit checkpoints and the gradient through an activation, in float64.

Between two FP8 linears of a stage (§2.1, §3.2 of the paper quantize each linear's own operands) a network has
    D = act(S + bias) + R          with S the product of the linear's codes, or
    H = act(G) * U                 with G, U the two projections of a gated feed-forward,
and its backward pass needs act' at the pre-activation, so the forward keeps it: in BF16, or in 8 bits as defined
by `pack`.  `gelu` is z Phi(z), `gelu_tanh` its tanh form, `silu` z / (1 + e^-z).
"""
from __future__ import annotations

import math

import numpy as np

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
GROUP = 32
_erf = np.vectorize(math.erf, otypes=[np.float64])


def _logistic(t):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-t))


def value(z, act: str) -> np.ndarray:
    z = np.asarray(z, dtype=np.float64)
    if act == "relu":
        return np.where(z < 0, 0.0, z)
    if act == "gelu":
        return z * 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * _logistic(z)
    return z


def slope(z, act: str) -> np.ndarray:
    z = np.asarray(z, dtype=np.float64)
    if act == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if act == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = _logistic(z)
        return p * (1.0 + z * (1.0 - p))
    return np.ones_like(z)


def gate(g, u, act: str) -> np.ndarray:
    return value(g, act) * np.asarray(u, dtype=np.float64)


def grad(dd, z, act: str) -> np.ndarray:
    return np.asarray(dd, dtype=np.float64) * slope(z, act)


def gate_grad(dd, g, u, act: str) -> np.ndarray:
    """dG and dU side by side."""
    dd = np.asarray(dd, dtype=np.float64)
    return np.concatenate([dd * np.asarray(u, dtype=np.float64) * slope(g, act), dd * value(g, act)], axis=1)


def pack(x):
    """(codes int8 [rows, cols], exponent bytes [rows, ceil(cols / 32)]) of float32 values.

    A group's step is 2^-s, s the largest integer <= 126 with amax 2^s <= 127; codes are x 2^s to nearest even and the byte
    is 127 - s.  The codes of the largest step (s = -122) stop at 63, so that they restore to finite float32 values.  A group
    with a NaN or an infinity: byte 255, codes 0.
    """
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    codes = np.zeros((rows, cols), dtype=np.int8)
    exps = np.zeros((rows, groups), dtype=np.uint8)
    for g in range(groups):
        part = x[:, g * GROUP:(g + 1) * GROUP]
        amax = np.abs(part).max(axis=1)
        fine = np.isfinite(part).all(axis=1)
        for r in range(rows):
            if not fine[r]:
                exps[r, g] = 255
                continue
            s = 126
            if amax[r] > 0.0:
                s = min(126, int(math.floor(math.log2(127.0 / amax[r]))) + 1)
                while amax[r] * 2.0 ** s > 127.0:
                    s -= 1
            exps[r, g] = 127 - s
            most = 63 if s == -122 else 127  # 64 steps of 2^122 are 2^128
            codes[r, g * GROUP:(g + 1) * GROUP] = np.clip(np.rint(part[r] * 2.0 ** s), -most, most).astype(np.int8)
    return codes, exps


def unpack(codes, exps) -> np.ndarray:
    codes, exps = np.asarray(codes, dtype=np.float64), np.asarray(exps, dtype=np.int64)
    step = np.where(exps == 255, np.nan, 2.0 ** (exps - 127.0))
    return codes * np.repeat(step, GROUP, axis=1)[:, :codes.shape[1]]
