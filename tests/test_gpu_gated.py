"""The dense gated block on the GPU, stage by stage against the oracle: every
stage is compared on the kernels' own saved inputs of that stage, so each
bound counts only that stage's roundings (bf16: 2^-8 of the value for each
rounding of a result; sums: the float32 rounding of at most K additions of
|a||b|, of which far fewer fall together)."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import dev, to_np
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
CODE = {"bf16": B.MOE_BF16, "f32": B.MOE_F32}
# the activations' exponential and reciprocal (about 1e-6) and a few roundings
ACT_EPS = 4e-6


def _problem(T, d, f, dt, pad=0, seed=0):
    rng = np.random.default_rng(seed + T + d + f)
    def t(rows, cols, std, extra=0):
        w = torch.from_numpy((rng.standard_normal((rows, cols + extra)) * std).astype(np.float32))
        return w.to(dev()).to(DT[dt])[:, :cols]
    return dict(x=t(T, d, 1, pad), w1=t(f, d, d ** -0.5).contiguous(), w3=t(f, d, d ** -0.5).contiguous(),
                w2=t(d, f, f ** -0.5).contiguous(), dy=t(T, d, 1, pad), add=t(T, d, 1, 2 * pad),
                dx_add=t(T, d, 1, pad))


def _sum_eps(K):
    """Rounding of a float32 sum of K products, relative to sum |a||b|: the
    matrix cores add them in a chain of at most K steps, half an ulp each; a random
    walk of those stays below 8 sqrt(K) of them."""
    return (8 * np.sqrt(K) + 4) * 2.0 ** -24


def _close(got, ref, bound, name):
    bad = np.abs(got - ref) > bound + 1e-30
    assert not bad.any(), (name, int(bad.sum()), np.abs(got - ref)[bad][:3], bound[bad][:3])


def _forward(P, act, dt, save=True, add=True, pad=0):
    T, d = P["x"].shape
    f = P["w1"].shape[0]
    y = torch.full((T + 1, d + pad), 5.0, dtype=DT[dt], device=dev())
    h = torch.empty(3, T, f, dtype=DT[dt], device=dev()) if save else None
    ws = B.workspace(B.moe_gated_ffn_fwd_workspace_bytes(CODE[dt], T, d, f), dev())
    B.moe_gated_ffn_fwd(B.ACTS[act], P["x"], P["w1"], P["w3"], P["w2"], y[:T, :d], ws,
                        add=P["add"] if add else None, h_save=h)
    assert (y[T:] == 5).all() and (y[:, d:] == 5).all()
    return y[:T, :d], h


SHAPES = [(1, 8, 8), (2, 64, 128), (7, 72, 200), (33, 136, 264), (130, 520, 392), (257, 256, 1032)]


@pytest.fixture(params=[0, 1, 2], ids=["auto", "tiles256", "tiles128"])
def tiles(request):
    B.moe_set_gemm_tiles(request.param)
    yield request.param
    B.moe_set_gemm_tiles(0)


# sizes at which the plan takes each kernel, tile height and split of K
LARGER = [(777, 40, 72), (1030, 40, 2056), (2056, 40, 2056), (2056, 1032, 72), (2056, 1032, 520), (4100, 40, 72),
          (4100, 40, 200), (4100, 136, 72), (4100, 136, 1032), (4100, 40, 2056), (777, 136, 2056),
          (1030, 1032, 2056), (4100, 1032, 1032), (4100, 1032, 2056), (200, 4104, 1032), (1, 2056, 72),
          (100, 40, 8200)]


@pytest.mark.parametrize("act", ["swiglu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f", SHAPES)
@pytest.mark.parametrize("pad", [0, 24])
def test_forward_and_backward(tiles, T, d, f, act, dt, pad):
    _check_block(T, d, f, act, dt, pad)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f", LARGER)
def test_every_plan(T, d, f, dt):
    _check_block(T, d, f, "swiglu", dt, 8)


def _check_block(T, d, f, act, dt, pad):
    P = _problem(T, d, f, dt, pad)
    N = {n: to_np(v) for n, v in P.items()}
    rnd = ROUND[dt]
    y, h = _forward(P, act, dt, pad=pad)
    f1, f3, a = to_np(h)
    H1, H3 = N["x"] @ N["w1"].T, N["x"] @ N["w3"].T
    e1, e3 = (_sum_eps(d) * (np.abs(N["x"]) @ np.abs(N[w]).T) for w in ("w1", "w3"))
    g, dg = O.gate_act(H1, act), O.gate_act_grad(H1, act)
    # |act'| < 1.13 and |act''| < 0.8 for all three, but ReLU's act' jumps where H1 may be on
    # either side of 0; near its zeros act' cancels, so its own error is that of terms up to 1 + |h|
    jump = (np.abs(H1) <= e1) if act == "relu" else 0
    _close(f3, g, (rnd + ACT_EPS) * np.abs(g) + 1.13 * e1, "act(H1)")
    _close(f1, H3 * dg, (rnd + ACT_EPS) * np.abs(H3 * dg) + np.abs(dg) * e3 * 1.01 +
           np.abs(H3) * (0.8 * e1 + ACT_EPS * (1 + np.abs(H1)) + jump), "H3 act'(H1)")
    _close(a, g * H3, (rnd + ACT_EPS) * np.abs(g * H3) + 1.13 * e1 * (np.abs(H3) + e3) + np.abs(g) * e3, "a")
    ref = N["add"] + a @ N["w2"].T
    _close(to_np(y), ref, rnd * np.abs(ref) + _sum_eps(f + 1) * (np.abs(N["add"]) + np.abs(a) @ np.abs(N["w2"]).T), "y")
    # without saved planes: the same bits
    y2, _ = _forward(P, act, dt, save=False, pad=pad)
    assert torch.equal(y, y2)

    for dw_dt in {DT[dt], torch.float32}:
        dx = torch.full((T + 1, d + pad), 5.0, dtype=DT[dt], device=dev())
        dw = [torch.full(s, 9.0, dtype=dw_dt, device=dev()) for s in ((f, d), (f, d), (d, f))]
        ws = B.workspace(B.moe_gated_ffn_bwd_workspace_bytes(CODE[dt], T, d, f), dev())
        B.moe_gated_ffn_bwd(B.ACTS[act], P["x"], h, P["w1"], P["w3"], P["w2"], P["dy"], dx[:T, :d], *dw, ws,
                            add=P["dx_add"])
        assert (dx[T:] == 5).all() and (dx[:, d:] == 5).all()
        b = O.gated_bwd(N["x"], f1, f3, a, N["w1"], N["w3"], N["w2"], N["dy"], N["dx_add"])
        rw = ROUND["bf16"] if dw_dt == torch.bfloat16 else 2.0 ** -24
        ref = b["dw2"]
        _close(to_np(dw[2]), ref, rw * np.abs(ref) + _sum_eps(T) * (np.abs(N["dy"]).T @ np.abs(a)), "dw2")
        # dH carries its own rounding and dA's sum
        eda = _sum_eps(d) * (np.abs(N["dy"]) @ np.abs(N["w2"]))
        e1 = (rnd + 2.0 ** -23) * np.abs(b["dh1"]) + eda * np.abs(f1)
        e3 = (rnd + 2.0 ** -23) * np.abs(b["dh3"]) + eda * np.abs(f3)
        ref = b["dx"]
        _close(to_np(dx)[:T, :d], ref, 1.01 * (rnd * np.abs(ref) + e1 @ np.abs(N["w1"]) + e3 @ np.abs(N["w3"]) +
               _sum_eps(2 * f) * (np.abs(b["dh1"]) @ np.abs(N["w1"]) + np.abs(b["dh3"]) @ np.abs(N["w3"]) +
                                  np.abs(N["dx_add"]))), "dx")
        for got, e, n in ((dw[0], e1, "1"), (dw[1], e3, "3")):
            ref = b["dw" + n]
            _close(to_np(got), ref, 1.01 * (rw * np.abs(ref) + (e + _sum_eps(T) * np.abs(b["dh" + n])).T @ np.abs(N["x"])), "dw" + n)


@pytest.mark.parametrize("T,d,f", [(9, 64, 96), (20, 8, 40)])
@pytest.mark.parametrize("act", ["swiglu", "gelu_tanh"])
def test_gradients_are_differences(T, d, f, act):
    """<gradient, v> against central differences of the float64 block along v."""
    P = _problem(T, d, f, "f32", seed=5)
    N = {n: to_np(v) for n, v in P.items()}
    y, h = _forward(P, act, "f32", add=False)
    dx = torch.empty(T, d, device=dev())
    dw = [torch.empty(s, device=dev()) for s in ((f, d), (f, d), (d, f))]
    B.moe_gated_ffn_bwd(B.ACTS[act], P["x"], h, P["w1"], P["w3"], P["w2"], P["dy"], dx, *dw,
                        B.workspace(B.moe_gated_ffn_bwd_workspace_bytes(B.MOE_F32, T, d, f), dev()))
    rng, step = np.random.default_rng(1), 1e-5
    ins = {n: N[n] for n in ("x", "w1", "w3", "w2")}
    for n, g in zip(ins, [dx, *dw]):
        v = rng.standard_normal(ins[n].shape)
        loss = [(O.gated_fwd(**dict(ins, **{n: ins[n] + s * step * v}), act=act)[3] * N["dy"]).sum() for s in (1, -1)]
        g = to_np(g)
        # the gradient's elements are within 1e-5 of their scale (as the float32 layer's are)
        tol = 1e-5 * (np.abs(g) + np.sqrt((g ** 2).mean())).ravel() @ np.abs(v).ravel() + 1e-6
        assert abs((loss[0] - loss[1]) / (2 * step) - (g * v).sum()) <= tol, n


def test_large_gate_values():
    """Pre-activations far out: the activation saturates, its gradient is 0 or 1 and never NaN."""
    for act in ("swiglu", "gelu_tanh", "relu"):
        T, d, f = 4, 8, 16
        x = torch.full((T, d), 1.0, device=dev())
        x[1] *= -1
        x[2] *= 1e18
        x[3] *= -1e18
        w1 = torch.ones(f, d, device=dev()) * 100
        w3, w2 = torch.ones(f, d, device=dev()) * 1e-20, torch.ones(d, f, device=dev())
        y, h = _forward(dict(x=x, w1=w1, w3=w3, w2=w2), act, "f32", add=False)
        dx = torch.empty(T, d, device=dev())
        dw = [torch.empty(s, device=dev()) for s in ((f, d), (f, d), (d, f))]
        B.moe_gated_ffn_bwd(B.ACTS[act], x, h, w1, w3, w2, torch.ones(T, d, device=dev()), dx, *dw,
                            B.workspace(B.moe_gated_ffn_bwd_workspace_bytes(B.MOE_F32, T, d, f), dev()))
        for t in (y, h, dx):
            assert torch.isfinite(t).all(), act
        # dW3 itself leaves float32's range here (dA act(h1) x = 8 * 8e20 * 1e18 = 6.4e39): an
        # infinity is right, a NaN would not be
        for t in dw:
            assert not torch.isnan(t).any(), act
        assert (y[1] == 0).all() and (y[3] == 0).all() and (y[0] > 0).all()


@pytest.mark.parametrize("act", ["swiglu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 70])
def test_a_token_that_is_not_a_number(tiles, T, dt, act):
    """Its output and its input gradient are NaN, and nobody else's."""
    P = _problem(T, 64, 72, dt)
    P["x"][1, 7] = float("nan")
    y, h = _forward(P, act, dt)
    dx = torch.empty(T, 64, dtype=DT[dt], device=dev())
    dw = [torch.empty(s, device=dev()) for s in ((72, 64), (72, 64), (64, 72))]
    B.moe_gated_ffn_bwd(B.ACTS[act], P["x"], h, P["w1"], P["w3"], P["w2"], P["dy"], dx, *dw,
                        B.workspace(B.moe_gated_ffn_bwd_workspace_bytes(CODE[dt], T, 64, 72), dev()))
    for t in (y, dx):
        bad = torch.isnan(t)
        assert bad[1].all() and bad.sum() == 64
    assert all(torch.isnan(w).all() for w in dw)


def test_no_tokens():
    T, d, f = 0, 16, 24
    P = _problem(T, d, f, "bf16")
    _forward(P, "swiglu", "bf16")
    for dt in (torch.bfloat16, torch.float32):
        dw = [torch.full(s, 9.0, dtype=dt, device=dev()) for s in ((f, d), (f, d), (d, f))]
        B.moe_gated_ffn_bwd(B.MOE_SWIGLU, P["x"], torch.empty(3, 0, f, dtype=torch.bfloat16, device=dev()),
                            P["w1"], P["w3"], P["w2"], P["dy"], torch.empty_like(P["dy"]), *dw,
                            B.workspace(B.moe_gated_ffn_bwd_workspace_bytes(B.MOE_BF16, T, d, f), dev()))
        assert all((w == 0).all() for w in dw)


def test_addend_may_be_the_output():
    P = _problem(40, 64, 72, "bf16")
    y, _ = _forward(P, "swiglu", "bf16", save=False)
    z = P["add"].clone()
    B.moe_gated_ffn_fwd(B.MOE_SWIGLU, P["x"], P["w1"], P["w3"], P["w2"], z,
                        B.workspace(B.moe_gated_ffn_fwd_workspace_bytes(B.MOE_BF16, 40, 64, 72), dev()), add=z)
    assert torch.equal(y.contiguous(), z)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f", [(40, 64, 72), (777, 520, 264), (777, 40, 2056), (2056, 1032, 520)])
def test_outputs_over_inputs(T, d, f, dt):
    """y over x, and dx over dy, x or the addend, with the bits of separate outputs (products
    whole and with K split)."""
    P = _problem(T, d, f, dt, pad=8)
    w, act = (P["w1"], P["w3"], P["w2"]), B.MOE_GELU_TANH
    y, h = _forward(P, "gelu_tanh", dt, add=False, pad=8)
    wider = lambda t: torch.cat([t, torch.full_like(t[:, :8], 3)], 1)
    x = wider(P["x"])
    B.moe_gated_ffn_fwd(act, x[:, :d], *w, x[:, :d],
                        B.workspace(B.moe_gated_ffn_fwd_workspace_bytes(CODE[dt], T, d, f), dev()))
    assert torch.equal(x[:, :d], y) and (x[:, d:] == 3).all()
    ws = B.workspace(B.moe_gated_ffn_bwd_workspace_bytes(CODE[dt], T, d, f), dev())

    def backward(**over):
        t = dict({n: wider(P[n])[:, :d] for n in ("x", "dy", "dx_add")})
        dx = t[over["dx"]] if over else torch.empty_like(P["x"])
        dw = [torch.empty_like(v) for v in w]
        B.moe_gated_ffn_bwd(act, t["x"], h, *w, t["dy"], dx, *dw, ws, add=t["dx_add"])
        return [dx] + dw
    want = backward()
    for n in ("dy", "x", "dx_add"):
        assert all(torch.equal(a, b) for a, b in zip(backward(dx=n), want)), n


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T", [12, 530])
def test_rows_as_far_apart_as_allowed(T, dt):
    """Rows 8 MB apart, so that offsets pass 32 bits: the bits of contiguous rows."""
    d, f, act = 72, 136, B.MOE_SWIGLU
    P = _problem(T, d, f, dt)
    w = (P["w1"], P["w3"], P["w2"])
    y, h = _forward(P, "swiglu", dt)
    ws = [B.workspace(q(CODE[dt], T, d, f), dev()) for q in (B.moe_gated_ffn_fwd_workspace_bytes,
                                                             B.moe_gated_ffn_bwd_workspace_bytes)]
    dx, dw = torch.empty_like(P["x"]), [torch.empty_like(v) for v in w]
    B.moe_gated_ffn_bwd(act, P["x"], h, *w, P["dy"], dx, *dw, ws[1], add=P["dx_add"])
    es = P["x"].element_size()
    far = torch.empty(T * ((1 << 23) - 64) // es, dtype=DT[dt], device=dev()).view(T, -1)
    V = {n: far[:, i * d:(i + 1) * d] for i, n in enumerate(("x", "dy", "add", "dx_add", "y", "dx"))}
    for n in ("x", "dy", "add", "dx_add"):
        V[n].copy_(P[n])
    h2, dw2 = torch.empty_like(h), [torch.empty_like(v) for v in w]
    B.moe_gated_ffn_fwd(act, V["x"], *w, V["y"], ws[0], add=V["add"], h_save=h2)
    B.moe_gated_ffn_bwd(act, V["x"], h2, *w, V["dy"], V["dx"], *dw2, ws[1], add=V["dx_add"])
    assert torch.equal(V["y"], y) and torch.equal(V["dx"], dx) and torch.equal(h2, h)
    assert all(torch.equal(a, b) for a, b in zip(dw, dw2))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f", [(1, 2056, 72), (40, 64, 72), (100, 40, 8200), (777, 136, 2056), (2056, 1032, 520)])
def test_workspace_is_all_that_is_written(T, d, f, dt):
    """The bytes behind a workspace of the queried size stay as they were."""
    P = _problem(T, d, f, dt)
    w = (P["w1"], P["w3"], P["w2"])

    def guarded(size):
        buf = torch.full((size + (1 << 20),), 77, dtype=torch.uint8, device=dev())
        return buf[:size], buf[size:]
    y, dx = torch.empty_like(P["x"]), torch.empty_like(P["x"])
    h, dw = torch.empty(3, T, f, dtype=DT[dt], device=dev()), [torch.empty_like(v) for v in w]
    ws, behind = guarded(B.moe_gated_ffn_fwd_workspace_bytes(CODE[dt], T, d, f))
    B.moe_gated_ffn_fwd(B.MOE_SWIGLU, P["x"], *w, y, ws)
    B.moe_gated_ffn_fwd(B.MOE_SWIGLU, P["x"], *w, y, ws, h_save=h)
    assert (behind == 77).all()
    ws, behind = guarded(B.moe_gated_ffn_bwd_workspace_bytes(CODE[dt], T, d, f))
    B.moe_gated_ffn_bwd(B.MOE_SWIGLU, P["x"], h, *w, P["dy"], dx, *dw, ws)
    assert (behind == 77).all()
