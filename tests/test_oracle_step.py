"""Pins of the oracle of the operators around the layer: closed forms, plain
torch on the CPU, automatic differentiation."""
import numpy as np
import pytest
import torch

import oracle as O


@pytest.mark.parametrize("rows,d", [(1, 8), (5, 40)])
def test_norm_and_its_gradients_are_torchs(rows, d):
    rng = np.random.default_rng(d)
    x, dy, ds = (rng.standard_normal((rows, d)) for _ in range(3))
    w, eps = rng.uniform(-2, 2, d), 2.0 ** -10
    s, r, y = O.rms_norm_fwd(x, w, eps)
    tx, tw = (torch.from_numpy(a).requires_grad_() for a in (x, w))
    ty = tx * torch.rsqrt(tx.square().mean(1, keepdim=True) + eps) * tw
    np.testing.assert_allclose(y, ty.detach().numpy(), rtol=1e-12)
    np.testing.assert_array_equal(s, x)
    gx, gw = torch.autograd.grad((ty * torch.from_numpy(dy)).sum() + (tx * torch.from_numpy(ds)).sum(), (tx, tw))
    dx, dw = O.rms_norm_bwd(s, r, w, dy, ds)
    np.testing.assert_allclose(dx, gx.numpy(), rtol=1e-11, atol=1e-13)
    np.testing.assert_allclose(dw, gw.numpy(), rtol=1e-11, atol=1e-13)


def test_norm_by_hand():
    s, r, y = O.rms_norm_fwd([[3.0, 4.0, 0.0, 0.0]], [1.0, 2.0, 1.0, 1.0], 2.0 ** -40)
    assert abs(r[0] - 0.4) < 1e-9 and np.allclose(y, [[1.2, 3.2, 0, 0]])
    # the addition rounds to the layer dtype before the norm: 1 + 2^-9 is 1 in bf16
    s, _, _ = O.rms_norm_fwd([[1.0, 1.0]], [1.0, 1.0], 0.1, add=[[2.0 ** -9, 2.0 ** -7]], dtype="bf16")
    assert s.tolist() == [[1.0, 1.0078125]]


def test_norm_rows_in_8_bits():
    rng = np.random.default_rng(5)
    x, w = rng.standard_normal((20, 64)).astype(np.float32), rng.uniform(0.5, 2, 64).astype(np.float32)
    s, r, y = O.rms_norm_fwd(x, w, 1e-5)
    q, scale = O.rms_norm_rows_i8(s, r, w)
    assert (np.abs(q * scale[:, None] - y) <= scale[:, None] * (0.5 + 1e-4)).all()
    assert (np.abs(q).max(axis=1) == 127).all()
