"""AdamW's 8-bit moments of an element whose v passes float32, in the oracle: its m does not outlive
its v."""
import numpy as np

import oracle as O

H = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8)


def test_codes_by_hand():
    none = np.zeros(6, np.int64)
    m, v = [1.0, -2.0, 1e20, -1e20, np.inf, 1e39], [1.0, 1e39, 4e40, 3e38, np.inf, np.inf]
    mc, me, vc, ve = O.adamw_encode_states(m, v, none, none)
    # -2 and 1e20 go with their v; the m of the finite v stays and is the block's largest; NaN stays
    assert me.tolist() == [193] and O.adamw_decode(mc, me, 3)[:4].tolist() == [0, 0, 0, -(2.0 ** 66) * 1.25]
    assert mc.tolist()[4:] == [128, 128]
    # (1, 16 octaves below, as the least code above 0)
    assert ve.tolist() == [254] and vc.tolist() == [1, 255, 255, 252, 255, 255]


def test_a_v_that_the_random_bits_round_past_float32():
    v = [2.0 ** 128 * (1 - 2.0 ** -7)] * 2          # half of the last code
    mc, me, vc, ve = O.adamw_encode_states([1.0, 1.0], v, np.zeros(2, np.int64), np.array([0, 65535]))
    assert vc.tolist() == [255, 255] and O.adamw_decode(mc, me, 3).tolist() == [1.0, 0.0]


def test_steps_after_an_overflow_are_of_ordinary_size():
    """One gradient of 1e21 in a block, and a whole block of them; then gradients of 1e-3 or 0.
    |m| / sqrt(v) <= (1 - b1) / sqrt((1 - b2) (1 - b1^2 / b2)) by Cauchy's inequality over any run of
    gradients; a step's codes are off by at most 1/8 in m and 1/16 in v, the sum of 4 steps' by
    (9/8)^4 in m and (15/16)^-4 in v: 1.82."""
    n, none = 256, np.zeros(256, np.int64)
    p, m, v = np.zeros(n), np.zeros(n), np.zeros(n)
    g = np.full(n, 1e-3)
    g[5] = 1e21
    g[128:] = -1e21
    most = 0.1 / np.sqrt(0.05 * (1 - 0.81 / 0.95)) * 1.82 * H["lr"] * (1 / (1 - 0.9 ** 100))
    for step in range(100, 105):
        before = p
        with np.errstate(over="ignore"):
            p, m, v = O.adamw(p, g, m, v, step=step, **H)
        assert (np.abs(p - before) <= most).all(), step
        mc, me, vc, ve = O.adamw_encode_states(m, v, none, none)
        m, v = O.adamw_decode(mc, me, 3), O.adamw_decode(vc, ve, 4)
        g = np.where(np.arange(n) % 2, 1e-3, 0.0)
