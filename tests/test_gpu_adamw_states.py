"""8-bit moments on the GPU of elements whose v passes float32: code for code as the oracle has them, and
the steps that follow."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import dev, to_np
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8)
HUGE = {5: 1e21, 6: -3e38, 77: 1e20, 130: np.inf, 131: np.nan, 140: 2e19, 141: -1e30, 511: 5e22}


@pytest.mark.parametrize("n", [512, 517, 2048 + 512])
def test_a_v_past_float32_takes_its_m_along(n):
    """Single ones, beside what is not finite, and a whole block; whole tiles and cut ones.

    p: with a v that is inf as float32 the update is 0; else as in 32 bits, 16 U of the update
    and 2 U of p.  The steps after: as the oracle's bound has it, |m| / sqrt(v) <=
    (1 - b1) / sqrt((1 - b2) (1 - b1^2 / b2)), times 1.82 for the codes' errors of 4 steps."""
    rng = np.random.default_rng(n)
    host = (rng.standard_normal(n) * 1e-3).astype(np.float32)
    for at, x in HUGE.items():
        host[at] = x
    host[256:384] = 1e25
    g = torch.from_numpy(host).to(dev())
    u8 = lambda k: torch.zeros(k, dtype=torch.uint8, device=dev())
    t = B.AdamWTensor(torch.ones(n, device=dev()), g, u8(n), u8(n), m_exp=u8(B.adamw_blocks(n)), v_exp=u8(B.adamw_blocks(n)))
    lst = B.AdamWList([t])
    odd = ~np.isfinite(host)
    p0, m, v = to_np(t.p), np.zeros(n), np.zeros(n)
    most = 0.1 / np.sqrt(0.05 * (1 - 0.81 / 0.95)) * 1.82 * H["lr"] / (1 - 0.9 ** 100)
    for step in range(100, 105):
        gr = to_np(g)
        B.moe_adamw(lst, **H, step=step, seed=step)
        rm, rv = O.adamw_random(n, step, 0)
        with np.errstate(over="ignore", invalid="ignore"):
            p, m, v = O.adamw(p0, gr, m, v, step=step, **H)
            p = np.where(np.isinf(v.astype(np.float32)) & ~odd, p0, p)
        got = to_np(t.p)
        assert np.isnan(got[odd]).all()
        size = np.abs(p - p0)[~odd]
        assert (np.abs(got - p)[~odd] <= 32 * U * size + 4 * U * np.abs(p0)[~odd]).all(), step
        assert (np.abs(got - p0)[~odd] <= most + 4 * U * np.abs(p0)[~odd]).all(), step
        codes = O.adamw_encode_states(m, v, rm, rv)
        for name, mine, want in zip(("m", "m_exp", "v", "v_exp"), (t.m, t.m_exp, t.v, t.v_exp), codes):
            np.testing.assert_array_equal(mine.cpu().numpy(), want, err_msg=f"{name} {step}")
        m, v, p0 = O.adamw_decode(*codes[:2], 3), O.adamw_decode(*codes[2:], 4), got
        g.copy_(torch.from_numpy(np.where(np.arange(n) % 2, rng.standard_normal(n) * 1e-3, 0.0).astype(np.float32)))
