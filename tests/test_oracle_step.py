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


def test_adamw_is_torchs():
    rng = np.random.default_rng(2)
    p, g1, g2 = (rng.standard_normal(50) for _ in range(3))
    t = torch.from_numpy(p.copy()).requires_grad_()
    opt = torch.optim.AdamW([t], lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    m = v = np.zeros(50)
    for step, g in enumerate((g1, g2), 1):
        t.grad = torch.from_numpy(g.copy())
        opt.step()
        p, m, v = O.adamw(p, g, m, v, 0.01, 0.9, 0.99, 1e-6, step, 0.1)
    np.testing.assert_allclose(p, t.detach().numpy(), rtol=1e-12)


def test_adamw_codes_by_hand():
    none = np.zeros(8, np.int64)
    # 1 is the top octave (exponent 127): codes count from 2^-15 (1 + 2^-k)
    c, e = O.adamw_encode([1.0, -1.0, 1.875, 1.124, 0.5, 2.0 ** -15 * 1.125, 2.0 ** -15, 0.0], none, 3)
    assert e.tolist() == [127] and c.tolist() == [120, 248, 127, 120, 112, 1, 0, 0]
    c, e = O.adamw_encode([1.0, 1.9375, 0.5, 2.0 ** -15, 1e-30, 0.0, 1.06, 0.75], none, 4)
    assert e.tolist() == [127] and c.tolist() == [240, 255, 224, 1, 1, 0, 240, 232]
    assert O.adamw_decode([1, 240, 0, 255], [127], 4).tolist() == [2.0 ** -15 * 1.0625, 1.0, 0.0, 1.9375]
    # 65535 of 65536: everything that is not on a code goes up, the largest past its octave
    c, e = O.adamw_encode([1.99, -1.01, 1.0, 0.0], np.full(4, 65535), 3)
    assert e.tolist() == [128] and O.adamw_decode(c, e, 3).tolist() == [2.0, -1.125, 1.0, 0.0]
    c, e = O.adamw_encode([np.nan, np.inf, 1e39, 1.0], none[:4], 3)
    assert e.tolist() == [127] and c.tolist() == [128, 128, 128, 120]
    c, e = O.adamw_encode([np.nan, np.inf, 1e39, 1.0], none[:4], 4)
    assert e.tolist() == [127] and c.tolist() == [255, 255, 255, 240]


@pytest.mark.parametrize("mant", [3, 4])
def test_adamw_every_code_comes_back(mant):
    for e in (16, 100, 254):
        code = np.arange(256).astype(np.uint8)
        if mant == 3:
            code[128] = 0
        # both blocks hold a value of the top octave
        code[0], code[255] = 127 if mant == 3 else 250, 255
        x = O.adamw_decode(code, [e, e], mant)
        c, ee = O.adamw_encode(x, np.zeros(256, np.int64), mant)
        assert ee.tolist() == [e, e] and (c == code).all()


@pytest.mark.parametrize("mant", [3, 4])
def test_adamw_rounding_is_right_on_average(mant):
    """Every value's mean over 2000 seeds, within 5 standard deviations of a step's uniform error."""
    rng = np.random.default_rng(4)
    x = np.exp(rng.uniform(-6, 0, 256)) * (rng.choice([-1, 1], 256) if mant == 3 else 1)
    tries = np.stack([O.adamw_decode(*O.adamw_encode(x, O.adamw_random(256, s, 3)[mant == 4], mant), mant)
                      for s in range(2000)])
    step = np.exp2(np.floor(np.log2(np.abs(x))) - mant)
    assert (np.abs(tries - x) <= step * 2).all()
    assert (np.abs(tries.mean(axis=0) - x) <= 5 * step / 2 / np.sqrt(2000)).all()


def test_adamw_random_bits():
    a, b = O.adamw_random(1 << 16, 7, 0)
    for r in (a, b):
        assert abs(r.mean() - 32767.5) < 5 * 65536 / np.sqrt(12 * 65536)
    assert (O.adamw_random(1 << 16, 8, 0)[0] != a).mean() > 0.99 and (O.adamw_random(1 << 16, 7, 1)[0] != a).mean() > 0.99
    np.testing.assert_array_equal(O.adamw_random(100, 7, 0, start=500)[1], b[500:600])
    big = O.adamw_random(4, 7, 0, start=(1 << 32) - 2)
    assert (big[0][2:] != a[:2]).any()


def test_vocab_loss_is_torchs():
    rng = np.random.default_rng(6)
    x, w = rng.standard_normal((7, 12)), rng.standard_normal((31, 12))
    t, c = np.array([0, 30, -1, 5, 5, -100, 31]), rng.uniform(0.5, 2, 7)
    o = O.vocab_loss(x, w, t, 0.25, c)
    tx, tw = (torch.from_numpy(a).requires_grad_() for a in (x, w))
    tt = torch.from_numpy(np.where(t == 31, -1, t)).clamp(min=-1)
    loss = torch.nn.functional.cross_entropy(tx @ tw.T, tt, ignore_index=-1, reduction="none")
    np.testing.assert_allclose(o["loss"], loss.detach().numpy(), rtol=1e-12, atol=1e-14)
    gx, gw = torch.autograd.grad((loss * torch.from_numpy(c) * 0.25).sum(), (tx, tw))
    np.testing.assert_allclose(o["dx"], gx.numpy(), rtol=1e-10, atol=1e-13)
    np.testing.assert_allclose(o["dw"], gw.numpy(), rtol=1e-10, atol=1e-13)
    assert (o["lse"][[2, 5, 6]] == 0).all()
    np.testing.assert_allclose(o["lse"][:2], torch.logsumexp(tx @ tw.T, 1).detach().numpy()[:2], rtol=1e-12)


def test_vocab_loss_by_hand():
    o = O.vocab_loss([[0.0, 0.0], [100.0, 0.0]], [[1.0, 0], [0, 1], [0, 0], [0, -1]], [1, 0])
    assert abs(o["loss"][0] - np.log(4)) < 1e-15 and np.allclose(o["dl"][0], [0.25, -0.75, 0.25, 0.25])
    assert 0 <= o["loss"][1] < 1e-40 and o["lse"][1] == 100
