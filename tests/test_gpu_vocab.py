"""The loss of a vocabulary projection and its gradients on the GPU against the oracle.

Tolerances.  U = 2^-24.  A product of n terms is summed in float32, at most 16 terms at a
time and n / 16 + 64 partial results in turn (steps, wavefronts, ranges): SUM(n) =
2 U (n / 16 + 64) of the sum of the terms' sizes.  A logit is off by at most D = SUM(d)
|x| |w|, a row's lse and loss by twice the largest D of the row, exponentials by a few U
times the distance from the maximum: 2e-6.  A probability is off by that, by half a step of
16 bits where it is kept in them (2^-11 relative, 2^-39 near 0), and dl by its rounding;
dx and dw by what dl's errors sum up to, their own sums, and one rounding."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import dev, to_np
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"bf16": B.MOE_BF16, "f32": B.MOE_F32}
ROUND = {"bf16": 2.0 ** -8, "f32": U}


def SUM(n):
    return 2 * U * (n / 16 + 64)


def _inputs(T, d, V, pad, dt, rng, ignored=0.2):
    w = rng.standard_normal((V, d)) * 3 / np.sqrt(d)
    t = rng.integers(0, V, T)
    x = rng.standard_normal((T, d)) + rng.uniform(0, 3, (T, 1)) * w[t]
    t = np.where(rng.random(T) < ignored, -1, t) if T > 1 else t
    wide = torch.full((T + 1, d + pad), 7.0, dtype=DT[dt], device=dev())
    wide[:T, :d] = torch.from_numpy(x.astype(np.float32)).to(dev())
    return wide[:T, :d], torch.from_numpy(w.astype(np.float32)).to(dev()).to(DT[dt]), t.astype(np.int32)


def _call(x, w, t, dt, grad, dw_dt=None, scale=1.0, weights=None, pad=0, ws=None):
    (T, d), V = x.shape, w.shape[0]
    full = lambda *s, v=5.0, t=torch.float32: torch.full(s, v, dtype=t, device=dev())
    o = dict(loss=full(T + 3), lse=full(T + 3), status=torch.zeros(1, dtype=torch.int32, device=dev()))
    if grad:
        o.update(dx=full(T + 1, d + pad, t=DT[dt]), dw=full(V + 1, d, t=DT[dw_dt or dt]))
    n = B.moe_vocab_loss_workspace_bytes(CODE[dt], T, d, V, CODE[dw_dt or dt] if grad else None)
    if ws is None:
        ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device=dev())       # (NaNs, as float32, bf16 and fp16)
    B.moe_vocab_loss(x, w, torch.from_numpy(t).to(dev()), o["loss"], o["lse"], o["status"], ws[:n] if n else ws,
                     scale=scale, weights=weights, dx=o["dx"][:T, :d] if grad else None, dw=o["dw"] if grad else None)
    torch.cuda.synchronize()
    assert (ws[n:] == 0xFF).all()
    return o


def _check(o, x, w, t, dt, dw_dt=None, scale=1.0, weights=None):
    T, d = x.shape
    X, W = to_np(x), to_np(w)
    r = O.vocab_loss(X, W, t, scale, weights)
    D = SUM(d) * np.abs(r["x"]) @ np.abs(W).T
    row = 2 * D.max(axis=1, initial=0) + 2e-6
    live = (t >= 0) & (t < len(W))
    for n in ("loss", "lse"):
        got = to_np(o[n])
        assert (np.abs(got[:T] - r[n]) <= row + 2 * U * (np.abs(r["lse"]) + 20)).all(), n
        assert (got[T:] == 5).all() and not got[:T][~live].any()
    if "dx" not in o:
        return
    c = np.abs(r["c"])[:, None]
    e = c * r["p"] * (row[:, None] + (2.0 ** -11 if dt == "bf16" else 0)) + c * 2.0 ** -39
    rows = np.nonzero(live)[0]
    # (the target's p - 1 comes from the loss)
    e[rows, t[rows]] = (c * (r["p"] * row[:, None] + 2 * U * (1 - r["p"])))[rows, t[rows]]
    e += ROUND[dt] * np.abs(r["dl"]) + 4 * U * c * r["p"]
    A = np.abs(r["dl"]) + e
    dx, dw = to_np(o["dx"]), to_np(o["dw"])
    bx = e @ np.abs(W) + SUM(len(W)) * A @ np.abs(W)
    bw = e.T @ np.abs(r["x"]) + SUM(T) * A.T @ np.abs(r["x"])
    assert (np.abs(dx[:T, :d] - r["dx"]) <= (1 + ROUND[dt]) * bx + ROUND[dt] * np.abs(r["dx"]) + 1e-40).all()
    assert (np.abs(dw[:-1] - r["dw"]) <= (1 + ROUND[dw_dt or dt]) * bw + ROUND[dw_dt or dt] * np.abs(r["dw"]) + 1e-40).all()
    assert not dx[:T, :d][~live].any()
    assert (dx[T:] == 5).all() and (dx[:, d:] == 5).all() and (dw[-1] == 5).all()


SIZES = [(1, 8, 1, 0), (1, 64, 7, 8), (1, 1024, 5003, 0), (2, 72, 8, 0), (3, 24, 9, 8), (5, 64, 129, 0), (15, 64, 1000, 0),
         (16, 520, 1003, 0), (17, 264, 1003, 8), (33, 128, 257, 0), (64, 1024, 4099, 0), (130, 64, 8191, 24),
         (300, 1024, 2050, 0), (509, 136, 3001, 64), (1030, 512, 5003, 0), (2049, 64, 511, 0)]
# the tiles of the products these do not take (test_vocab_plans): bf16, then float32
TILES = {"bf16": [(497, 592, 32682), (20, 328, 138), (356, 72, 11443), (230, 200, 26644), (2698, 64, 3153), (331, 80, 29154),
                  (22, 2040, 149), (1481, 1296, 2329), (71, 536, 19796)],
         "f32": [(44, 64, 37519), (329, 64, 12709), (238, 72, 25045), (1494, 64, 6065), (525, 80, 18553), (38, 72, 34014),
                 (395, 1832, 5237), (19, 224, 26377), (1642, 1184, 165)]}


@pytest.mark.parametrize("dt,T,d,V", [(dt, *s) for dt in TILES for s in TILES[dt]])
def test_tiles(dt, T, d, V):
    x, w, t = _inputs(T, d, V, 0, dt, np.random.default_rng(V))
    _check(_call(x, w, t, dt, True), x, w, t, dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,V,pad", SIZES)
def test_loss(dt, T, d, V, pad):
    x, w, t = _inputs(T, d, V, pad, dt, np.random.default_rng(T + d + V))
    _check(_call(x, w, t, dt, False), x, w, t, dt)


@pytest.mark.parametrize("dt,dw_dt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("T,d,V,pad", SIZES)
def test_gradients(dt, dw_dt, T, d, V, pad):
    rng = np.random.default_rng(T * d + V)
    x, w, t = _inputs(T, d, V, pad, dt, rng)
    c = rng.uniform(0, 2, T).astype(np.float32)
    kw = dict(dw_dt=dw_dt, scale=1 / 64)
    _check(_call(x, w, t, dt, True, pad=pad, weights=torch.from_numpy(c).to(dev()), **kw), x, w, t, dt, weights=c, **kw)
    _check(_call(x, w, t, dt, True, **kw), x, w, t, dt, **kw)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("mode", [1, 2])
def test_other_tiles(dt, mode):
    """256 x 256 and 128-column tiles at sizes that take others by themselves."""
    try:
        B.moe_set_gemm_tiles(mode)
        for T, d, V in ((5, 64, 129), (300, 264, 2051), (700, 512, 1000)):
            x, w, t = _inputs(T, d, V, 0, dt, np.random.default_rng(V))
            _check(_call(x, w, t, dt, False), x, w, t, dt)
            _check(_call(x, w, t, dt, True), x, w, t, dt)
    finally:
        B.moe_set_gemm_tiles(0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T", [7, 300])
def test_ignored_and_bad_targets(dt, T):
    """Nothing of an ignored row comes through, NaN and infinities included; a target beyond the
    vocabulary is ignored and sets its bit."""
    d, V = 72, 1003
    rng = np.random.default_rng(T)
    x, w, t = _inputs(T, d, V, 0, dt, rng)
    t[:6] = [-1, 5, -100, V, 2 ** 31 - 1, -2 ** 31]
    clean = x.clone()
    clean[[0, 2, 3, 4, 5]] = 0
    for row, v in ((0, np.nan), (2, np.inf), (3, np.nan), (4, -np.inf), (5, 3e38)):
        x[row] = v
    for grad in (False, True):
        o = _call(x, w, t, dt, grad)
        assert o["status"].item() == B.STATUS_BAD_TARGET
        _check(o, clean, w, t, dt)
    t[3:5] = -1
    assert _call(x, w, t, dt, True)["status"].item() == 0
    t[:] = -1                                   # every token ignored
    o = _call(x, w, t, dt, True)
    assert not o["loss"][:T].any() and not o["dx"][:T].any() and not o["dw"][:V].any()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_that_are_not_finite_stay_their_own(dt):
    d, V = 64, 300
    x, w, t = _inputs(40, d, V, 0, dt, np.random.default_rng(0), ignored=0)
    x[3, 5], x[17] = np.nan, np.inf
    odd = torch.tensor([i in (3, 17) for i in range(40)], device=dev())
    for grad in (False, True):
        o = _call(x, w, t, dt, grad)
        assert o["loss"][:40][odd].isnan().all() and o["loss"][:40][~odd].isfinite().all()
        if grad:
            assert o["dx"][:40][odd].isnan().all() and o["dx"][:40][~odd].isfinite().all()
            assert o["dw"][:V].isnan().any()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 200])
def test_extreme_logits(dt, T):
    """Logits of hundreds: targets with all of the probability and with none."""
    d, V = 64, 1000
    rng = np.random.default_rng(T)
    w = torch.from_numpy(np.sign(rng.standard_normal((V, d))).astype(np.float32)).to(dev()).to(DT[dt])
    t = rng.integers(0, V, T).astype(np.int32)
    x = w[torch.from_numpy(t).long().to(dev())] * 8              # the target's logit is 512, exactly
    other = (t + 1) % V
    for target in (t, other.astype(np.int32)):
        o = _call(x, w, target, dt, True)
        _check(o, x, w, target, dt)
        if target is t:
            assert (o["loss"][:T] >= 0).all() and (o["loss"][:T] < 1e-30).all()
        else:
            assert (o["loss"][:T] > 100).all()


@pytest.mark.parametrize("dt,dw_dt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_pieces(dt, dw_dt):
    """More tokens than a piece holds, the last one shorter: the sums of dw carry over.  Against
    torch in 64 bits on the device, a block of rows at a time."""
    T, d, V = (40000, 16, 65541) if dt == "bf16" else (20000, 16, 65541)
    assert T * V * (2 if dt == "bf16" else 4) > 2 ** 32
    x, w, t = _inputs(T, d, V, 0, dt, np.random.default_rng(1), ignored=0.1)
    o = _call(x, w, t, dt, True, dw_dt=dw_dt, scale=1 / 16)
    tt = torch.from_numpy(t).to(dev()).long()
    W = w.double()
    dw, size = torch.zeros(V, d, dtype=torch.float64, device=dev()), torch.zeros(V, d, dtype=torch.float64, device=dev())
    step = ROUND[dt]
    for r0 in range(0, T, 2500):
        rows = slice(r0, r0 + 2500)
        live = (tt[rows] >= 0)[:, None]
        X = x[rows].double() * live
        l = X @ W.T
        lse = torch.logsumexp(l, 1)
        at = tt[rows].clamp(min=0)[:, None]
        loss = torch.where(live[:, 0], lse - l.gather(1, at)[:, 0], 0.0)
        row = 2 * SUM(d) * (X.abs() @ W.abs().T).amax(1, keepdim=True) + 2e-6
        assert ((o["loss"][:T][rows].double() - loss).abs() <= row[:, 0] + 2 * U * (lse.abs() + 20)).all()
        # dl's errors as in _check, the target's too
        p = torch.exp(l - lse[:, None]) * live / 16
        e = p * (row + 4 * U + (2.0 ** -11 if dt == "bf16" else 0)) + 2.0 ** -43
        dl = p.scatter_add(1, at, (live / -16.0).double())
        e += step * dl.abs()
        A = dl.abs() + e
        dx, bound = dl @ W, e @ W.abs() + SUM(V) * A @ W.abs()
        got = o["dx"][:T, :d][rows].double()
        assert ((got - dx).abs() <= (1 + step) * bound + step * dx.abs()).all()
        dw += dl.T @ X
        size += e.T @ X.abs() + SUM(T) * A.T @ X.abs()
    last = ROUND[dw_dt]
    assert ((o["dw"][:V].double() - dw).abs() <= (1 + last) * size + last * dw.abs()).all()
    assert (o["dw"][V] == 5).all()


def test_many_rows_of_the_loss_alone():
    """More rows than one piece of maxima and sums holds."""
    T, d, V = 70000, 16, 65541
    assert T * (V // 128) * 8 > 2 ** 28
    x, w, t = _inputs(T, d, V, 0, "bf16", np.random.default_rng(2), ignored=0.1)
    o = _call(x, w, t, "bf16", False)
    for r0 in (0, 30000, T - 2000):
        rows = slice(r0, r0 + 2000)
        r = O.vocab_loss(to_np(x[rows]), to_np(w), t[rows])
        np.testing.assert_allclose(to_np(o["loss"][:T][rows]), r["loss"], rtol=0, atol=1e-4)


def test_in_place_and_no_tokens():
    x, w, t = _inputs(300, 64, 1000, 8, "bf16", np.random.default_rng(0))
    o = _call(x, w, t, "bf16", True)
    ws = B.workspace(B.moe_vocab_loss_workspace_bytes(B.MOE_BF16, 300, 64, 1000, B.MOE_BF16), dev())
    dw, loss = torch.empty_like(w), torch.empty(300, device=dev())
    B.moe_vocab_loss(x, w, torch.from_numpy(t).to(dev()), loss, None, o["status"], ws, dx=x, dw=dw)   # over x, lse left out
    assert torch.equal(x, o["dx"][:300, :64]) and torch.equal(dw, o["dw"][:1000]) and torch.equal(loss, o["loss"][:300])
    e = torch.empty(0, device=dev())
    B.moe_vocab_loss(x[:0], w, torch.empty(0, dtype=torch.int32, device=dev()), e, e, o["status"], ws, dx=x[:0], dw=dw)
    assert not dw.any()


def test_gradients_are_the_losses_differences():
    """Central differences of the kernel's own loss: logits of a few units, truncation h^2 |w|^3 / 6 below
    1e-4, roundings of a loss of 8 (1e-6) over 2 h."""
    T, d, V, h = 4, 16, 50, 1e-2
    x, w, t = _inputs(T, d, V, 0, "f32", np.random.default_rng(9), ignored=0)
    x = x.contiguous()
    o = _call(x, w, t, "f32", True)
    f = lambda x, w: _call(x, w, t, "f32", False)["loss"][:T].double().sum().item()
    for k in range(0, T * d, 3):
        e = torch.zeros(T * d, device=dev())
        e[k] = h
        e = e.view(T, d)
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - o["dx"][:T, :d].reshape(-1)[k].item()) < 1e-3
    for k in range(0, V * d, 17):
        e = torch.zeros(V * d, device=dev())
        e[k] = h
        e = e.view(V, d)
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - o["dw"][:V].reshape(-1)[k].item()) < 1e-3


@pytest.mark.parametrize("T,grad", [(3, False), (200, True), (900, True)])
def test_captured_and_replayed(T, grad):
    d, V = 128, 3001
    rng = np.random.default_rng(T)
    x, w, t = _inputs(T, d, V, 0, "bf16", rng)
    x, t = x.contiguous(), torch.from_numpy(t).to(dev())
    out = lambda: dict(loss=torch.empty(T, device=dev()), lse=torch.empty(T, device=dev()),
                       dx=torch.empty_like(x), dw=torch.empty_like(w))
    status = torch.zeros(1, dtype=torch.int32, device=dev())
    n = B.moe_vocab_loss_workspace_bytes(B.MOE_BF16, T, d, V, B.MOE_BF16 if grad else None)

    def step(o, ws):
        B.moe_vocab_loss(x, w, t, o["loss"], o["lse"], status, ws, scale=1 / T, dx=o["dx"] if grad else None,
                         dw=o["dw"] if grad else None)

    a, b, ws = out(), out(), B.workspace(n, dev())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, ws)
    for k in range(4):
        nx, _, nt = _inputs(T, d, V, 0, "bf16", rng)
        x.copy_(nx)
        t.copy_(torch.from_numpy(nt))
        graph.replay()
        step(b, B.workspace(n, dev()))
        torch.cuda.synchronize()
        for name in (a if grad else ("loss", "lse")):
            assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("T", [3, 40])
def test_weights_past_32_bits(T):
    """A vocabulary whose weights (and dW) reach past 2^31 elements and 2^32 bytes."""
    d, V = 4104, 530000
    assert V * d > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(T)
    w = torch.empty(V, d, dtype=torch.bfloat16, device=dev())
    for part in w.split(50000):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * 3 / d ** 0.5)
    x = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
    t = torch.randint(V - 1000, V, (T,), generator=g, device="cuda")
    t[0] = 5
    o = _call(x, w, t.int().cpu().numpy(), "bf16", T > 16)
    X = x.double()
    l = torch.cat([X @ part.double().T for part in w.split(50000)], 1)
    lse = torch.logsumexp(l, 1)
    loss = lse - l.gather(1, t[:, None])[:, 0]
    # D: the sum of 4104 products' sizes is at most |x| |w| (Cauchy), 1.2 * 64 * 3.2
    D = 2 * SUM(d) * 1.2 * 64 * 3.2 + 2e-6 + 2 * U * 40
    assert (o["loss"][:T].double() - loss).abs().max() <= D and (o["lse"][:T].double() - lse).abs().max() <= D
    if T > 16:
        p = torch.exp(l - lse[:, None])
        dl = p.scatter_add(1, t[:, None], torch.full((T, 1), -1.0, dtype=torch.float64, device="cuda"))
        e = p * (D + 2.0 ** -11) + 2.0 ** -8 * dl.abs() + 2.0 ** -39
        for rows in (slice(0, 2000), slice(V // 2, V // 2 + 2000), slice(V - 2000, V)):
            dw = dl[:, rows].T @ X
            bound = (e[:, rows].T + SUM(T) * dl[:, rows].abs().T) @ X.abs()
            assert ((o["dw"][:V][rows].double() - dw).abs() <= 1.01 * bound + 2.0 ** -8 * dw.abs()).all()
        dx, dxe = 0, 0
        for part, q, r in zip(w.split(50000), dl.split(50000, 1), e.split(50000, 1)):
            W = part.double()
            dx, dxe = dx + q @ W, dxe + r @ W.abs() + SUM(V) * q.abs() @ W.abs()
        assert ((o["dx"][:T, :d].double() - dx).abs() <= 1.01 * dxe + 2.0 ** -8 * dx.abs()).all()
