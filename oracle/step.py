"""Oracle of the operators around the layer in a training step and in int8
serving: the root-mean-square norm, the loss of the vocabulary projection, and
the AdamW step.  Plain numpy in float64, straight from the formulas in
include/moe.h; roundings are left to the caller except where the formula has
one."""
from __future__ import annotations

import numpy as np

from .blocks import quantize_rows
from .moe_oracle import round_to

__all__ = ["rms_norm_fwd", "rms_norm_bwd", "rms_norm_rows_i8"]


# ---- norm ------------------------------------------------------------------------
def rms_norm_fwd(x, weight, eps, add=None, dtype="f32"):
    """(s, r, y): s = x + add rounded to the layer dtype (x + add in float32
    first, as the sum of two values of that type is), y unrounded."""
    s = np.asarray(x, np.float64)
    if add is not None:
        s = round_to((s + np.asarray(add, np.float64)).astype(np.float32).astype(np.float64), dtype)
    with np.errstate(invalid="ignore", over="ignore"):
        r = 1 / np.sqrt((s * s).mean(axis=1) + float(np.float32(eps)))
        return s, r, s * r[:, None] * np.asarray(weight, np.float64)


def rms_norm_rows_i8(s, r, weight):
    """(q, scale): a = s weight in float32, q and c as quantize_rows forms them of
    a, scale = c r."""
    with np.errstate(invalid="ignore", over="ignore"):
        a = (np.asarray(s, np.float64) * np.asarray(weight, np.float64)).astype(np.float32)
    q, c = quantize_rows(a)
    return q, c.astype(np.float64) * r


def rms_norm_bwd(s, r, weight, dy, dsum=None):
    """(dx, dw)."""
    g = dy * weight
    dx = r[:, None] * (g - s * (r * r * (g * s).mean(axis=1))[:, None])
    return dx if dsum is None else dx + dsum, (dy * s * r[:, None]).sum(axis=0)
