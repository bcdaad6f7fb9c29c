"""The shared expert and the int8 experts inside MoELayer: against the routed
layer and the oracle, in every forward that takes them, in a captured graph and
on a stream of its own."""
import numpy as np
import pytest
import torch

import oracle as O
import workloads as W
from gpu_util import RTOL, assert_close, dev, to_dev, to_np, torch_dtype
from paper_2205_01848_amd import MoELayer, QuantizedExperts, binding as B, rows_alloc_for

pytestmark = pytest.mark.gpu

CAP = ("dynamic", 21, 20)


def _setup(dt, act, T=300, d=136, E=5, f=200, sf=104, sact="swiglu", backward=True, seed=0):
    wl = W.small("c5", T=T, d=d, E=E, f=f, act=act, dtype=dt, name=f"blocks{seed}", x_std=8.0)
    I = W.make_inputs(wl)
    dv = {n: to_dev(getattr(I, n), dt) for n in ("x", "w_g", "w1", "w3", "w2", "dy")}
    dv["bias"] = to_dev(I.bias, "f32")
    rng = np.random.default_rng(seed)
    mk = lambda *s: torch.from_numpy((rng.standard_normal(s) * s[1] ** -0.5).astype(np.float32)).to(dev()).to(torch_dtype(dt))
    dv["shared"] = (mk(sf, d), mk(sf, d), mk(d, sf))
    R = rows_alloc_for(*CAP[:1], T, wl.k, E, *CAP[1:])
    L = MoELayer(T, d, E, wl.k, f, act, torch_dtype(dt), R, backward=backward, shared_f=sf, shared_act=sact)
    return wl, dv, L


def _gate(dv, wl):
    return dict(w_g=dv["w_g"], bias=dv["bias"], renorm=wl.renorm, capacity=CAP)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act,sact", [("swiglu", "swiglu"), ("gelu_tanh", "gelu_tanh"), ("relu", "relu")])
def test_shared_expert_in_training(dt, act, sact):
    wl, dv, L = _setup(dt, act, sact=sact)
    w = dv["w1"], dv["w3"], dv["w2"]
    routed = L.forward(dv["x"], *w, **_gate(dv, wl)).clone()
    droute = L.backward(dv["x"], dv["dy"], *w, w_g=dv["w_g"], renorm=wl.renorm).clone()
    dw1 = L.dw1.clone()
    y = L.forward(dv["x"], *w, **_gate(dv, wl), shared=dv["shared"])
    dx = L.backward(dv["x"], dv["dy"], *w, w_g=dv["w_g"], renorm=wl.renorm, shared=dv["shared"])
    assert torch.equal(dw1, L.dw1)              # the routed experts' part is the same
    s = [to_np(t) for t in dv["shared"]]
    x, dy = to_np(dv["x"]), to_np(dv["dy"])
    f1, f3, a, ref = O.gated_fwd(x, *s, sact, to_np(routed))
    b = O.gated_bwd(x, f1, f3, a, *s, dy, to_np(droute))
    # the layer's own tolerance: a few roundings to the layer dtype along the way
    assert_close(to_np(y), ref, RTOL[dt], "y")
    assert_close(to_np(dx), b["dx"], RTOL[dt], "dx")
    for n in ("1", "3", "2"):
        assert_close(to_np(getattr(L, "dsw" + n)), b["dw" + n], RTOL[dt], "dsw" + n)


def test_shared_expert_in_every_forward():
    """The fused forward, the separate steps, the cached one: the same bits."""
    wl, dv, L = _setup("bf16", "swiglu", backward=False)
    w = dv["w1"], dv["w3"], dv["w2"]
    y = L.forward(dv["x"], *w, **_gate(dv, wl), shared=dv["shared"]).clone()
    ids, weights = L.ids.clone(), L.weights.clone()
    L.combine = type(L).combine.__get__(L)       # a step of the instance's own: called one by one
    assert torch.equal(y, L.forward(dv["x"], *w, **_gate(dv, wl), shared=dv["shared"]))
    del L.combine
    assert torch.equal(y, L.forward(dv["x"], *w, ids=ids, weights=weights, capacity=CAP, shared=dv["shared"]))
    out, unchanged = torch.empty_like(ids), torch.zeros(1, dtype=torch.int32, device=dev())
    z = L.forward_cached(dv["x"], *w, cached=ids, cache_out=out, unchanged=unchanged, **_gate(dv, wl),
                         shared=dv["shared"])
    assert torch.equal(y, z)


def test_refusals():
    wl, dv, L = _setup("bf16", "swiglu", backward=False)
    w = dv["w1"], dv["w3"], dv["w2"]
    plain = MoELayer(wl.T, wl.d, wl.E, wl.k, wl.f, "swiglu", torch.bfloat16, L.rows_alloc)
    with pytest.raises(ValueError, match="shared_f"):
        plain.forward(dv["x"], *w, **_gate(dv, wl), shared=dv["shared"])
    with pytest.raises(ValueError, match="shape"):
        L.forward(dv["x"], *w, **_gate(dv, wl), shared=tuple(t[:-8] for t in dv["shared"]))
    q = QuantizedExperts(*(t[:-1].contiguous() for t in w))
    with pytest.raises(ValueError, match="sizes"):
        L.forward_i8(dv["x"], q, **_gate(dv, wl))


def _i8_bound(L, dv, q, wl, act, dt):
    """(y, bound) of the routed int8 layer from the routing it chose: each kept
    pick's expert output within ffn_i8_bounds and its rounding, combined."""
    dest, wts = L.dest_row.cpu().numpy(), L.weights.cpu().numpy().astype(np.float64)
    off, fill = L.offsets.cpu().numpy(), L.fill.cpu().numpy()
    xq, xs = O.quantize_rows(to_np(dv["x"]))
    src = L.src.cpu().numpy()
    rnd = 2.0 ** -8 if dt == "bf16" else 2.0 ** -24
    Y, B_ = np.zeros((L.rows_alloc, wl.d)), np.zeros((L.rows_alloc, wl.d))
    n = lambda a, e, w: None if a is None else a[e].cpu().numpy()[..., :w] if w else a[e].cpu().numpy()
    for e in range(wl.E):
        r = np.arange(off[e], off[e] + fill[e])
        if len(r) == 0:
            continue
        t = src[r] // wl.k
        y, slack = O.ffn_i8_bounds(xq[t], xs[t], n(q.w1, e, wl.d), n(q.s1, e, 0), n(q.w3, e, wl.d), n(q.s3, e, 0),
                                   n(q.w2, e, wl.f), n(q.s2, e, 0), act, dt)
        Y[r], B_[r] = y, slack * 1.001 + np.abs(y) * (rnd + 4 * 2.0 ** -24)
    out, bound = np.zeros((wl.T, wl.d)), np.zeros((wl.T, wl.d))
    for j in range(wl.k):
        kept = dest[:, j] >= 0
        out[kept] += wts[kept, j, None] * Y[dest[kept, j]]
        bound[kept] += wts[kept, j, None] * (B_[dest[kept, j]] + np.abs(Y[dest[kept, j]]) * 2.0 ** -22)
    return out, bound + rnd * (np.abs(out) + bound)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["swiglu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("T,E,f,cap", [(1, 5, 200, CAP), (300, 5, 200, CAP), (90, 33, 72, ("static", 1, 2)),
                                       (700, 4, 264, ("dynamic", 1, 1))])
def test_int8_layer(dt, act, T, E, f, cap):
    wl, dv, L = _setup(dt, act, T=T, E=E, f=f, backward=False)
    if cap[0] == "static":
        L = MoELayer(T, wl.d, E, wl.k, f, act, torch_dtype(dt), rows_alloc_for(cap[0], T, wl.k, E, *cap[1:]))
    q = QuantizedExperts(dv["w1"], dv["w3"], dv["w2"])
    y = to_np(L.forward_i8(dv["x"], q, **dict(_gate(dv, wl), capacity=cap)))
    assert L.status.item() == 0
    ref, bound = _i8_bound(L, dv, q, wl, act, dt)
    assert (np.abs(y - ref) <= bound + 1e-30).all()
    # the same routing given as cached picks, on the separate dispatch: the same bits
    ids, weights = L.ids.clone(), L.weights.clone()
    z = L.forward_i8(dv["x"], q, ids=ids, weights=weights, capacity=cap)
    assert (to_np(z) == y).all()
    z = L.forward_i8(dv["x"], q, ids=ids, weights=weights, capacity=("policy", 1, 1))
    assert (to_np(z) == y).all()


def test_int8_layer_with_shared_expert_is_near_the_real_layer():
    """Served in int8 against the bf16 layer on the same weights: within the
    quantisation (8 bits of weights, tokens and hidden values: a few percent)."""
    wl, dv, L = _setup("bf16", "swiglu", T=512, d=256, f=512, sf=128, backward=False)
    w = dv["w1"], dv["w3"], dv["w2"]
    y = to_np(L.forward(dv["x"], *w, **_gate(dv, wl), shared=dv["shared"]))
    z = to_np(L.forward_i8(dv["x"], QuantizedExperts(*w), **_gate(dv, wl), shared=dv["shared"]))
    assert np.linalg.norm(y - z) < 0.05 * np.linalg.norm(y)
    assert np.linalg.norm(y - z) > 0


def test_no_tokens():
    wl, dv, _ = _setup("bf16", "swiglu")
    L = MoELayer(0, wl.d, wl.E, wl.k, wl.f, "swiglu", torch.bfloat16, 8, backward=True, shared_f=104)
    x = torch.empty(0, wl.d, dtype=torch.bfloat16, device=dev())
    w = dv["w1"], dv["w3"], dv["w2"]
    L.forward(x, *w, **_gate(dv, wl), shared=dv["shared"])
    L.backward(x, x, *w, w_g=dv["w_g"], renorm=wl.renorm, shared=dv["shared"])
    L.forward_i8(x, QuantizedExperts(*w), **_gate(dv, wl), shared=dv["shared"])
    torch.cuda.synchronize()
    assert not L.dsw1.any() and not L.dsw2.any() and not L.dsw3.any()


@pytest.mark.parametrize("serve", [False, True])
def test_graph_and_stream(serve):
    """A step captured once, replayed on changed inputs with eager work between, and the
    same step on another stream: the eager step's bits."""
    wl, dv, L = _setup("bf16", "swiglu", T=260, sf=200)
    w = dv["w1"], dv["w3"], dv["w2"]
    q = QuantizedExperts(*w)
    xs = [dv["x"], dv["x"].flip(0).contiguous(), dv["dy"]]
    x, dy = dv["x"].clone(), dv["dy"]

    def step():
        if serve:
            L.forward_i8(x, q, **_gate(dv, wl), shared=dv["shared"])
        else:
            L.forward(x, *w, **_gate(dv, wl), shared=dv["shared"])
            L.backward(x, dy, *w, w_g=dv["w_g"], renorm=wl.renorm, shared=dv["shared"])

    def snap():
        torch.cuda.synchronize()
        return [getattr(L, n).clone() for n in ["y"] + ([] if serve else ["dx", "dw1", "dsw1", "dsw3", "dsw2"])]

    eager = []
    for v in xs:
        x.copy_(v)
        step()
        eager.append(snap())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x.copy_(xs[0])
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(snap(), eager[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in (1, 2, 0, 1):
        x.copy_(xs[turn])
        L.y.fill_(7)
        graph.replay()
        got = snap()
        assert all(torch.equal(a, b) for a, b in zip(got, eager[turn])), turn
        step()                                   # eager work in between
        assert all(torch.equal(a, b) for a, b in zip(snap(), eager[turn]))
