"""Pins of the oracle of the int8 products and the dense gated block: hand
cases, plain torch on the CPU, automatic differentiation and differences."""
import numpy as np
import pytest
import torch

import oracle as O

ACTS = ["swiglu", "gelu_tanh", "relu"]


def test_quantize_by_hand():
    x = np.array([[127.0, -127.0, 0.5, 1.5, 2.5, -0.5, 126.5, 0.0],     # scale 1: ties to even
                  [0.0] * 8,
                  [254.0, 1.0, 3.0, 5.0, -3.0, 2.0, 0.9, 1.1]])         # scale 2
    q, s = O.quantize_rows(x)
    assert s.tolist() == [1.0, 0.0, 2.0]
    assert q[0].tolist() == [127, -127, 0, 2, 2, 0, 126, 0]
    assert not q[1].any()
    assert q[2].tolist() == [127, 0, 2, 2, -2, 1, 0, 1]


def test_quantize_marks_rows_that_are_not_finite():
    q, s = O.quantize_rows(np.array([[1.0, np.nan], [np.inf, 1.0], [-np.inf, np.inf], [1.0, 2.0]]))
    assert np.isnan(s[:3]).all() and not q[:3].any()
    assert s[3] == np.float32(2.0) * (np.float32(1) / np.float32(127))


def test_quantize_is_within_half_a_step():
    x = np.random.default_rng(0).standard_normal((50, 301)).astype(np.float32).astype(np.float64)
    q, s = O.quantize_rows(x)
    assert (np.abs(q * s[:, None].astype(np.float64) - x) <= s[:, None] * (0.5 + 1e-12)).all()
    assert (np.abs(q).max(axis=1) == 127).all()


def test_matmul_is_the_scaled_whole_number_product():
    rng = np.random.default_rng(1)
    xq, wq = rng.integers(-127, 128, (5, 40)), rng.integers(-127, 128, (7, 40))
    xs, ws = rng.random(5), rng.random(7)
    ref = [[xs[r] * ws[n] * sum(int(a) * int(b) for a, b in zip(xq[r], wq[n])) for n in range(7)]
           for r in range(5)]
    np.testing.assert_allclose(O.matmul_i8(xq, xs, wq, ws), ref, rtol=1e-14)


def _block(seed, T=6, d=8, f=16):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal(s) for s in ((T, d), (f, d), (f, d), (d, f), (T, d), (T, d))]


@pytest.mark.parametrize("act", ACTS)
def test_gated_block_is_autograd(act):
    x, w1, w3, w2, dy, add = _block(2)
    t = [torch.tensor(a, requires_grad=True) for a in (x, w1, w3, w2)]
    F = torch.nn.functional
    g = {"swiglu": F.silu, "relu": F.relu, "gelu_tanh": lambda h: F.gelu(h, approximate="tanh")}[act]
    y = torch.tensor(add) + (g(t[0] @ t[1].T) * (t[0] @ t[2].T)) @ t[3].T
    y.backward(torch.tensor(dy))
    f1, f3, a, got = O.gated_fwd(x, w1, w3, w2, act, add)
    np.testing.assert_allclose(got, y.detach().numpy(), rtol=1e-12, atol=1e-12)
    b = O.gated_bwd(x, f1, f3, a, w1, w3, w2, dy, add)
    for name, ref in zip(("dx", "dw1", "dw3", "dw2"), t):
        r = ref.grad.numpy() + (add if name == "dx" else 0)
        np.testing.assert_allclose(b[name], r, rtol=1e-11, atol=1e-12)


@pytest.mark.parametrize("act", ["swiglu", "gelu_tanh"])
def test_gated_gradients_are_differences(act):
    x, w1, w3, w2, dy, _ = _block(3)
    ins = dict(x=x, w1=w1, w3=w3, w2=w2)
    f1, f3, a, _ = O.gated_fwd(x, w1, w3, w2, act)
    b = O.gated_bwd(x, f1, f3, a, w1, w3, w2, dy)
    rng, step = np.random.default_rng(4), 1e-5
    for name in ins:
        v = rng.standard_normal(ins[name].shape)
        loss = [(O.gated_fwd(**dict(ins, **{name: ins[name] + s * step * v}), act=act)[3] * dy).sum()
                for s in (1, -1)]
        assert abs((loss[0] - loss[1]) / (2 * step) - (b["d" + name] * v).sum()) < 1e-7 * (
            1 + abs((b["d" + name] * v).sum()))


@pytest.mark.parametrize("act", ACTS)
def test_int8_ffn_is_near_the_real_one(act):
    """The quantised FFN against the FFN of the values it stands for, and its slack is small."""
    rng = np.random.default_rng(5)
    R, d, f = 9, 64, 96
    q = lambda *s: O.quantize_rows(rng.standard_normal(s))
    (xq, xs), (w1, s1), (w3, s3), (w2, s2) = q(R, d), q(f, d), q(f, d), q(d, f)
    y, slack = O.ffn_i8_bounds(xq, xs, w1, s1, w3, s3, w2, s2, act, "bf16")
    val = lambda a, s: a * s[:, None].astype(np.float64)
    h1, h3 = val(xq, xs) @ val(w1, s1).T, val(xq, xs) @ val(w3, s3).T
    a = O.gate_act(h1, act) * h3 if act == "swiglu" else O.act_fwd(h1, act)
    ref = a @ val(w2, s2).T
    # A's 8 bits: at most half a step of each of its f values, and a bf16 rounding
    bound = (np.abs(a).max(axis=1)[:, None] / 127 * 0.51 + np.abs(a) * 2.0 ** -8) @ np.abs(val(w2, s2)).T
    assert (np.abs(y - ref) <= bound).all()
    assert np.median(slack) < 0.05 * np.median(bound)


# largest bf16 values of a row, up to a power of two, whose product with the float32 nearest
# to 1/127 is not the rounded quotient
OTHER_MAXIMA = (143, 144, 175, 207, 208, 239)


def test_the_scale_is_the_product():
    """The header's scale, max|x| times float32(1/127), and not max|x| / 127 rounded; half the
    largest value lies next to 63.5 scales and shows which of the two is meant."""
    m = np.arange(128, 256).astype(np.float32)
    x = np.zeros((128, 8))
    x[:, 0], x[:, 1], x[:, 2] = m, m / 2, -m / 2
    q, s = O.quantize_rows(x)
    assert (s == m * (np.float32(1) / np.float32(127))).all()
    assert tuple(m[s != m / np.float32(127)]) == OTHER_MAXIMA
    by_product = np.rint(m / 2 / s.astype(np.float64))
    by_quotient = np.rint(m / 2 / (m / np.float32(127)).astype(np.float64))
    assert (q[:, 1] == by_product).all() and (q[:, 2] == -by_product).all()
    assert set(m[by_product != by_quotient]) <= set(OTHER_MAXIMA) and (by_product != by_quotient).any()
