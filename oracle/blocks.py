"""Oracle of the feed-forward blocks beside the layer's own experts: rows in
8-bit integers and the products on them, and the dense gated block.  Plain
numpy in float64, straight from the formulas in include/moe.h; roundings are
left to the caller except where the formula has one (the int8 values, their
float32 scale, A in the layer dtype)."""
from __future__ import annotations

import numpy as np

from .moe_oracle import act_fwd, act_grad, round_to

__all__ = ["quantize_rows", "matmul_i8", "gate_act", "gate_act_grad", "gated_fwd", "gated_bwd",
           "ffn_i8_bounds"]


def quantize_rows(x: np.ndarray):
    """(q, scale): scale = max|x| times the float32 nearest to 1/127, as
    float32, q = rint(x / scale), ties to even, in [-127, 127].  A non-finite
    row: scale NaN, q 0."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        amax = np.abs(x).max(axis=1)
    fine = np.isfinite(amax)
    # max |x| is a float32 value; the product is rounded once
    scale = np.where(fine, amax, 0.0).astype(np.float32) * (np.float32(1) / np.float32(127))
    live = fine & (scale > 0)
    q = np.zeros(x.shape, dtype=np.int8)
    q[live] = np.clip(np.rint(x[live] / scale[live, None].astype(np.float64)), -127, 127)
    return q, np.where(fine, scale, np.float32(np.nan)).astype(np.float32)


def matmul_i8(xq, xs, wq, ws):
    """y[r, n] = xs[r] ws[n] sum_k xq[r, k] wq[n, k] for one expert."""
    acc = np.asarray(xq, np.float64) @ np.asarray(wq, np.float64).T   # whole numbers below 2^53: exact
    return acc * np.asarray(xs, np.float64)[:, None] * np.asarray(ws, np.float64)


def gate_act(h, act):
    return h / (1 + np.exp(-h)) if act == "swiglu" else act_fwd(h, act)


def gate_act_grad(h, act):
    if act == "swiglu":
        g = 1 / (1 + np.exp(-h))
        return g * (1 + h * (1 - g))
    return act_grad(h, act)


def gated_fwd(x, w1, w3, w2, act, add=None):
    """(H3 act'(H1), act(H1), A, Y) of the dense gated block."""
    h1, h3 = x @ w1.T, x @ w3.T
    g = gate_act(h1, act)
    a = g * h3
    y = a @ w2.T
    return h3 * gate_act_grad(h1, act), g, a, y if add is None else add + y


def gated_bwd(x, f1, f3, a, w1, w3, w2, dy, add=None):
    """dict of dH1, dH3, dX, dW1, dW3, dW2 from the planes of gated_fwd."""
    da = dy @ w2
    dh1, dh3 = da * f1, da * f3
    dx = dh1 @ w1 + dh3 @ w3
    return dict(dh1=dh1, dh3=dh3, dx=dx if add is None else add + dx, dw1=dh1.T @ x, dw3=dh3.T @ x,
                dw2=dy.T @ a)


def ffn_i8_bounds(xq, xs, w1, s1, w3, s3, w2, s2, act, dtype):
    """(y, slack) of one expert's int8 FFN.

    A is rounded to the layer dtype and then to 8 bits, so where A (known to a
    relative error eps in float32) lies next to a border, either value is
    right.  slack bounds what that can change: for every element the 8-bit
    value's distance over the interval A (1 +- eps), the scale's own interval
    included, through |W2|.

    eps: H is a whole number times two float32 factors (3 roundings).  The
    activation is h g(z) with g the logistic function, z = h (swiglu) or
    1.6 h (1 + 0.045 h^2) (GELU): a relative error of z changes g by that times
    |z| (1 - g), and z carries those 3 roundings (cubed for GELU) and about 4
    of its own; about 8 more roundings follow."""
    u = 2.0 ** -24
    h = matmul_i8(xq, xs, w1, s1)
    if act == "swiglu":
        a = gate_act(h, act) * matmul_i8(xq, xs, w3, s3)
    else:
        a = act_fwd(h, act)
    z = {"relu": 0 * h, "swiglu": h,
         "gelu_tanh": 2 * np.sqrt(2 / np.pi) * (h + 0.044715 * h ** 3)}[act]
    eps = u * (16 + 16 * np.abs(z) / (1 + np.exp(np.minimum(z, 700))))
    lo, hi = (round_to(a - np.abs(a) * eps, dtype), round_to(a + np.abs(a) * eps, dtype))
    mid = round_to(a, dtype)
    small = np.minimum(np.abs(lo), np.abs(hi)).max(axis=1) / 127
    large = np.maximum(np.abs(lo), np.abs(hi)).max(axis=1) / 127
    q, scale = quantize_rows(mid)
    value = q * scale[:, None].astype(np.float64)
    off = np.zeros_like(a)
    for s in (small * (1 - 2 * u), large * (1 + 2 * u)):
        s1d = np.where(s > 0, s, 1)[:, None]
        for v in (lo, hi):
            off = np.maximum(off, np.abs(np.clip(np.rint(v / s1d), -127, 127) * s[:, None] - value))
    w = np.asarray(w2, np.float64) * np.asarray(s2, np.float64)[:, None]
    return value @ w.T, off @ np.abs(w).T
