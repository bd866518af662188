"""8-bit layers in 64 bits: rows to codes, the scaled product, the seam between two blocks.  Written from the
definitions in include/flashbon_ops.h; numpy only.
"""
from __future__ import annotations

import numpy as np

from oracle.dit import gelu_tanh

TINY = np.float32(2.0 ** -126)
NONE, LAYER, RMS = 0, 1, 2


def quant_rows(v):
    """(codes int8 [M][K], scales float32 [M]) of rows v; ties to even; rows that are not finite: scale NaN, codes 0."""
    v = np.asarray(v, np.float64)
    with np.errstate(all="ignore"):
        scale = np.maximum((np.abs(v).max(1) / 127.0).astype(np.float32), TINY)
        bad = ~np.isfinite(scale)
        q = np.rint(v / np.where(bad, np.float32(1), scale).astype(np.float64)[:, None])
    q[bad] = 0
    scale[bad] = np.nan
    return q.astype(np.int8), scale


def linear(a, a_scale, w, w_scale, bias=None):
    """a_scale w_scale (a w^T) + bias; the whole-number product is exact (below 2^31)."""
    acc = np.asarray(a, np.float64) @ np.asarray(w, np.float64).T
    v = acc * np.asarray(a_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64)
    return v if bias is None else v + np.asarray(bias, np.float64)


def linear_gelu(*args):
    return gelu_tanh(linear(*args))


def norm(v, kind, eps):
    v = np.asarray(v, np.float64)
    if kind == NONE:
        return v
    if kind == LAYER:
        v = v - v.mean(1, keepdims=True)
    return v / np.sqrt((v * v).mean(1, keepdims=True) + eps)


def seam(x, y, alpha, post, gain, gate, pre, shift, scale, eps):
    """(h float64, a float64): a is the next block's norm of h as it is stored, in fp32."""
    one = lambda t, d: d if t is None else np.asarray(t, np.float64)  # noqa: E731
    eps = float(np.float32(eps))
    h = float(np.float32(alpha)) * np.asarray(x, np.float64)
    if y is not None:
        h = h + one(gate, 1.0) * (norm(y, post, eps) * one(gain, 1.0))
    a = norm(h.astype(np.float32), pre, eps) * (1.0 + one(scale, 0.0)) + one(shift, 0.0)
    return h, a
