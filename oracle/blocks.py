"""FP8 with a scale for each block of 128, products of such operands, and the norms around a residual sum with their
gradients, in float64.

A finer form of the casts and products of §2.1 and §3.2 of the paper, whose scales are per tensor: a block is 128 columns
of `block_rows` rows, and its scale a power of two by the same rule (the largest e with max |x| 2^e <= fmax).
"""
from __future__ import annotations

import numpy as np

from oracle import fp8
from oracle.scaling import scale_exponent

BLOCK = 128


def pack(x, fmt, block_rows: int = 1):
    """(codes uint8 [rows, cols], exponent bytes [ceil(rows / block_rows), ceil(cols / 128)]) of float values.

    A block's e is the largest integer <= 126 with max |x| 2^e <= fmax (126 for zeros; never below -120), its byte 127 - e, its
    codes x 2^e to nearest even.  A block with a NaN or an infinity: byte 255, codes 0x7F.
    """
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    codes = np.zeros((rows, cols), dtype=np.uint8)
    exps = np.zeros((-(-rows // block_rows), -(-cols // BLOCK)), dtype=np.uint8)
    for i in range(exps.shape[0]):
        for b in range(exps.shape[1]):
            at = np.s_[i * block_rows:(i + 1) * block_rows, b * BLOCK:(b + 1) * BLOCK]
            part = x[at]
            if not np.isfinite(part).all():
                exps[i, b], codes[at] = 255, 0x7F
                continue
            a = float(np.abs(part).max())
            e = 126 if a == 0.0 else scale_exponent(a, fmt, 0)
            exps[i, b] = 127 - e
            codes[at] = fp8.encode(part * 2.0 ** e, fmt)
    return codes, exps


def unpack(codes, exps, fmt, block_rows: int = 1) -> np.ndarray:
    exps = np.asarray(exps, dtype=np.int64)
    step = np.where(exps == 255, np.nan, 2.0 ** (exps - 127.0))
    rows, cols = np.asarray(codes).shape
    return fp8.decode(codes, fmt) * np.repeat(np.repeat(step, block_rows, 0)[:rows], BLOCK, 1)[:, :cols]


def rstd(v, eps):
    v = np.asarray(v, dtype=np.float64)
    return 1.0 / np.sqrt((v * v).mean(1) + eps)


def _gates(gate, gate_rows, rows):
    return 1.0 if gate is None else np.repeat(np.asarray(gate, np.float64), min(gate_rows, rows), 0)[:rows]


def residual(x, y, *, x_scale=1.0, y_scale=1.0, post=None, post_eps=None, gate=None, gate_rows=1):
    """r = x_scale x + y_scale gate p, p = y rstd(y) post, or y where post_eps is None.  x or y may be None; post: the
    effective weight (offset included)."""
    r = 0.0 if x is None else x_scale * np.asarray(x, np.float64)
    if y is not None:
        p = np.asarray(y, np.float64)
        if post_eps is not None:
            p = p * rstd(p, post_eps)[:, None] * (1.0 if post is None else post)
        r = r + y_scale * _gates(gate, gate_rows, p.shape[0]) * p
    return r


def norm(r, eps, weight=None):
    r = np.asarray(r, np.float64)
    return r * rstd(r, eps)[:, None] * (1.0 if weight is None else weight)


def norm_grad(d, v, eps):
    """The gradient of v rstd(v), given d, that of the product."""
    f = rstd(v, eps)[:, None]
    n = v * f
    return f * (d - n * (d * n).mean(1, keepdims=True))


def residual_grad(dr, dh, r, y, *, x_scale=1.0, y_scale=1.0, post=None, post_eps=None, pre=None, pre_eps=None, gate=None,
                  gate_rows=1):
    """Gradients of x, y, post, pre and gate; those that do not exist are None."""
    out = dict(dx=None, dy=None, dpost=None, dpre=None, dgate=None)
    t = 0.0 if dr is None else np.asarray(dr, np.float64)
    if dh is not None:
        dh, r = np.asarray(dh, np.float64), np.asarray(r, np.float64)
        out["dpre"] = (dh * r * rstd(r, pre_eps)[:, None]).sum(0)
        t = t + norm_grad(dh * (1.0 if pre is None else pre), r, pre_eps)
    out["dx"] = x_scale * t
    if y is None:
        return out
    y = np.asarray(y, np.float64)
    rows = y.shape[0]
    m = y if post_eps is None else y * rstd(y, post_eps)[:, None]
    w = 1.0 if post is None or post_eps is None else post
    b = y_scale * t
    if gate is not None:
        s = b * m * w
        out["dgate"] = np.stack([s[g * gate_rows:(g + 1) * gate_rows].sum(0) for g in range(-(-rows // gate_rows))])
    d = b * _gates(gate, gate_rows, rows)
    out["dpost"] = (d * m).sum(0)
    out["dy"] = d if post_eps is None else norm_grad(d * w, y, post_eps)
    return out
