"""Oracle of the operators around the layer in a training step and in int8
serving: the root-mean-square norm, the loss of the vocabulary projection, and
the AdamW step.  Plain numpy in float64, straight from the formulas in
include/moe.h; roundings are left to the caller except where the formula has
one."""
from __future__ import annotations

import numpy as np

from .blocks import quantize_rows
from .moe_oracle import round_to

__all__ = ["rms_norm_fwd", "rms_norm_bwd", "rms_norm_rows_i8", "vocab_loss", "adamw", "adamw_random", "adamw_encode",
           "adamw_encode_states", "adamw_decode"]


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


# ---- loss of a vocabulary projection ---------------------------------------------
def vocab_loss(x, w, targets, scale=1.0, weights=None):
    """dict of loss, lse, p (probabilities), dl, dx, dw; rows of ignored tokens (targets outside the
    vocabulary) are zeros in all but p."""
    t = np.asarray(targets)
    live = (t >= 0) & (t < len(w))
    x = np.where(live[:, None], np.asarray(x, np.float64), 0.0)
    l = x @ np.asarray(w, np.float64).T
    top = l.max(axis=1)
    z = np.exp(l - top[:, None])
    logs = np.log(z.sum(axis=1))
    p = z / z.sum(axis=1, keepdims=True)
    at = np.where(live, t, 0)
    rows = np.arange(len(t))
    c = np.where(live, scale * (1.0 if weights is None else np.asarray(weights, np.float64)), 0.0)
    loss = np.where(live, logs + (top - l[rows, at]), 0.0)
    dl = p * c[:, None]
    dl[rows, at] = c * np.expm1(-loss)
    return dict(loss=loss, lse=np.where(live, top + logs, 0.0), p=p, c=c, dl=dl, dx=dl @ np.asarray(w, np.float64),
                dw=dl.T @ x, x=x)


# ---- AdamW -----------------------------------------------------------------------
def adamw(p, g, m, v, lr, beta1, beta2, eps, step, weight_decay=0.0):
    """(p, m, v) after one step, unrounded."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * (g * g)
    with np.errstate(invalid="ignore", over="ignore"):
        p = p - lr * (weight_decay * p + m / (1 - beta1 ** step) / (np.sqrt(v / (1 - beta2 ** step)) + eps))
    return p, m, v


def adamw_random(n, seed, tensor, start=0):
    """The 16 random bits for m and the 16 for v of elements start .. start + n - 1 of the list's
    tensor number `tensor`."""
    u = np.uint32
    i = np.arange(start, start + n, dtype=np.uint64)
    lo, hi = (i & 0xFFFFFFFF).astype(u), (i >> 32).astype(u)
    with np.errstate(over="ignore"):
        key = u(seed & 0xFFFFFFFF) ^ u((tensor + 1) * 0x9E3779B9 & 0xFFFFFFFF)
        h = lo * u(0xBB67AE85) + hi * u(0x6A09E667) + key
        h = (h ^ (h >> u(16))) * u(0x9E3779B1)
        h = (h ^ (h >> u(15))) * u(0x85157AF5)
        h ^= h >> u(16)
    return (h & u(0xFFFF)).astype(np.int64), (h >> u(16)).astype(np.int64)


def _blocks(a, fill):
    out = np.full(-(-len(a) // 128) * 128, fill, dtype=a.dtype)
    out[:len(a)] = a
    return out.reshape(-1, 128)


def _steps(x, rnd, mant):
    """(some, octave, steps, beyond): whether a value is a number other than 0, its float32 exponent and
    its 2^-mant of that octave, the random 16 bits deciding on the one begun, and whether that is
    no finite float32."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        size = np.abs(x)
        some = np.isfinite(size) & (size > 0)
        frac, octave = np.frexp(np.where(some, size, 1.0))        # frac in [1/2, 1)
        steps = np.floor(frac * 2 ** (mant + 1) + rnd / 65536).astype(np.int64)   # 2^mant .. 2^(mant+1)
        octave = octave.astype(np.int64) - 1 + 127                # the float32 exponent
    carry = steps == 2 ** (mant + 1)
    octave, steps = octave + carry, np.where(carry, 2 ** mant, steps)
    return some, octave, steps, ~np.isfinite(size) | (some & (octave > 254))


def adamw_encode(x, rnd, mant):
    """(code, exponent per block) of values in float64: m (mant 3, with sign) or v (mant 4)."""
    x = np.asarray(x, np.float64)
    some, octave, steps, beyond = _steps(x, rnd, mant)
    e = np.maximum(_blocks(np.where(some & ~beyond, octave, 16), 16).max(axis=1), 16)
    top = np.repeat(e, 128)[:len(x)]
    code = (octave - (top - 15)) * 2 ** mant + steps - 2 ** mant
    code = np.where(some & (code > 0), code, 0)
    if mant == 3:
        code = np.where(beyond, 128, np.where((code > 0) & (x < 0), code + 128, code))
    else:
        code = np.where(beyond, 255, np.where((code == 0) & some, 1, code))
    return code.astype(np.uint8), e.astype(np.uint8)


def adamw_encode_states(m, v, rnd_m, rnd_v):
    """(code of m, its exponents, code of v, its exponents).  An m beside a v beyond float32, which
    no code stands for, is kept as 0."""
    lost = _steps(v, rnd_v, 4)[3] & ~_steps(m, rnd_m, 3)[3]
    return adamw_encode(np.where(lost, 0.0, m), rnd_m, 3) + adamw_encode(v, rnd_v, 4)


def adamw_decode(code, e, mant):
    c = np.asarray(code, np.int64)
    size = c & 127 if mant == 3 else c
    octave = np.repeat(np.asarray(e, np.int64), 128)[:len(c)] - 15 + size // 2 ** mant
    x = np.where(size > 0, (1 + size % 2 ** mant / 2 ** mant) * 2.0 ** (octave - 127.0), 0.0)
    return np.where(c == 128, np.nan, np.where(c > 128, -x, x)) if mant == 3 else x
