"""The operators around the layer together, as a model uses them: a training step (norm with
the residual's addition, layer, norm, vocabulary loss, their backward, AdamW) against plain torch
in 64 bits, the same step captured in a graph, and a serving step (norm with rows in 8 bits into
the layer's int8 forward)."""
import numpy as np
import pytest
import torch

from gpu_util import assert_close, dev, to_np
from paper_2205_01848_amd import AdamW, MoELayer, QuantizedExperts, RMSNorm, VocabLoss, rows_alloc_for
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

T, d, E, k, f, V = 300, 64, 4, 2, 96, 501
EPS = 1e-5


class Model:
    """One block: h = x + a, y = layer(norm(h)) + shared(norm(h)), logits of norm(h + y)."""

    def __init__(self, dtype, bits=32, captured=False):
        g = torch.Generator().manual_seed(11)
        r = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dev()).to(dtype)
        self.w = dict(g1=1 + r(d, std=0.1), g2=1 + r(d, std=0.1), w_g=r(E, d, std=0.3), w1=r(E, f, d, std=0.15),
                      w3=r(E, f, d, std=0.15), w2=r(E, d, f, std=0.15), s1=r(f, d, std=0.15), s3=r(f, d, std=0.15),
                      s2=r(d, f, std=0.15), head=r(V, d, std=0.2))
        self.norm1, self.norm2 = (RMSNorm(T, d, dtype, EPS, backward=True) for _ in "12")
        self.layer = MoELayer(T, d, E, k, f, "swiglu", dtype, rows_alloc_for("exact", T, k, E), backward=True, shared_f=f)
        self.loss = VocabLoss(T, d, V, dtype, backward=True)
        w, L = self.w, self.layer
        self.names = ["w1", "w3", "w2", "w_g", "s1", "s3", "s2", "g1", "g2", "head"]
        pairs = L.gradients(w["w1"], w["w3"], w["w2"], w_g=w["w_g"], shared=(w["s1"], w["s3"], w["s2"]))
        pairs += [(w["g1"], self.norm1.dw), (w["g2"], self.norm2.dw), (w["head"], self.loss.dw)]
        assert [p.data_ptr() for p, _ in pairs] == [w[n].data_ptr() for n in self.names]
        self.grads = {n: g for n, (_, g) in zip(self.names, pairs)}
        self.opt = AdamW(pairs, lr=0.01, bits=bits, captured=captured, min_8bit=1000)

    def gradients(self, x, a, targets):
        w, L = self.w, self.layer
        shared = (w["s1"], w["s3"], w["s2"])
        n1 = self.norm1.forward(x, w["g1"], add=a)
        y = L.forward(n1, w["w1"], w["w3"], w["w2"], w_g=w["w_g"], renorm=1, shared=shared)
        n2 = self.norm2.forward(self.norm1.sum, w["g2"], add=y)
        self.loss.forward(n2, w["head"], targets)
        dh2 = self.norm2.backward(self.loss.dx, w["g2"])               # reaches the stream and the layer alike
        dn1 = L.backward(n1, dh2, w["w1"], w["w3"], w["w2"], w_g=w["w_g"], renorm=1, shared=shared)
        return self.norm1.backward(dn1, w["g1"], dsum=dh2)

    def step(self, x, a, targets):
        dx = self.gradients(x, a, targets)
        self.opt.apply()
        return dx


def _batch(seed, dtype):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(V, (T,), generator=g).int()
    t[torch.rand(T, generator=g) < 0.1] = -1
    x, a = (torch.randn(T, d, generator=g).to(dev()).to(dtype) for _ in "xa")
    return x, a, t.to(dev())


def _reference(w, x, a, targets, ids):
    """Loss and gradients in 64 bits on the CPU, with the layer's picks."""
    w = {n: t.detach().double().cpu().requires_grad_() for n, t in w.items()}
    x = x.double().cpu().requires_grad_()
    t, ids = targets.long().cpu(), ids.long().cpu()
    rms = lambda s, g: s * (s.square().mean(1, keepdim=True) + EPS).rsqrt() * g
    silu = torch.nn.functional.silu
    h = x + a.double().cpu()
    n = rms(h, w["g1"])
    p = torch.softmax(n @ w["w_g"].T, 1).gather(1, ids)
    p = p / p.sum(1, keepdim=True)
    y = (silu(n @ w["s1"].T) * (n @ w["s3"].T)) @ w["s2"].T
    for e in range(E):
        one = (silu(n @ w["w1"][e].T) * (n @ w["w3"][e].T)) @ w["w2"][e].T
        y = y + one * (p * (ids == e)).sum(1, keepdim=True)
    logits = rms(h + y, w["g2"]) @ w["head"].T
    loss = torch.nn.functional.cross_entropy(logits, t, ignore_index=-1, reduction="none")
    names = list(w)
    g = torch.autograd.grad(loss.sum() / T, [x] + [w[n] for n in names])
    return loss.detach().numpy(), dict(zip(["x"] + names, (v.numpy() for v in g)))


def test_training_step():
    """Ten stages, each within the repository's 1e-5 for float32: 1e-4."""
    m = Model(torch.float32)
    x, a, t = _batch(0, torch.float32)
    before = {n: w.clone() for n, w in m.w.items()}
    dx = m.gradients(x, a, t)
    loss, g = _reference(before, x, a, t, m.layer.ids)
    assert_close(to_np(m.loss.loss), loss, 1e-4, "loss")
    assert_close(to_np(dx), g["x"], 1e-4, "dx")
    for n in m.names:
        assert_close(to_np(m.grads[n]), g[n].reshape(m.grads[n].shape), 1e-4, n)
    # the step itself, from those gradients, as torch's AdamW in 64 bits does it
    params = {n: before[n].double().cpu().requires_grad_() for n in m.names}
    ref = torch.optim.AdamW([dict(params=[params[n]], weight_decay=0.1 if params[n].dim() > 1 else 0.0) for n in m.names],
                            lr=0.01, betas=(0.9, 0.95), eps=1e-8)
    for n in m.names:
        params[n].grad = m.grads[n].double().cpu().reshape(params[n].shape)
    m.opt.step()
    ref.step()
    for n in m.names:
        # (two roundings of the weight, and 16 of an update of lr and less)
        p = params[n].detach().numpy()
        assert (np.abs(to_np(m.w[n]) - p) <= 2.0 ** -24 * (2 * np.abs(p) + 2 * np.abs(to_np(before[n])) + 20 * 0.01)).all(), n


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 32), (torch.bfloat16, 32), (torch.bfloat16, 8)])
def test_captured_steps(dtype, bits):
    """A captured step replayed on other batches, with its schedule sent to the device, and eager work
    between the replays, leaves the weights and states of eager steps bit for bit."""
    eager, cap = Model(dtype, bits), Model(dtype, bits, captured=True)
    x, a, t = _batch(0, dtype)
    keep = [w.clone() for w in cap.w.values()] + [s.clone() for s in _states(cap)]
    cap.opt.prepare()
    cap.opt.step_count = 0
    cap.step(x, a, t)                    # (what is allocated on first use)
    for now, was in zip([*cap.w.values(), *_states(cap)], keep):
        now.copy_(was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dx = cap.step(x, a, t)
    for k in range(1, 5):
        nx, na, nt = _batch(k, dtype)
        for to, new in ((x, nx), (a, na), (t, nt)):
            to.copy_(new)
        cap.opt.prepare(lr=0.01 / k)
        graph.replay()
        eager.opt.prepare(lr=0.01 / k)
        ref = eager.step(nx, na, nt)
        torch.cuda.synchronize()
        assert torch.equal(dx, ref) and torch.equal(cap.loss.loss, eager.loss.loss)
        for n in eager.names:
            assert torch.equal(cap.w[n], eager.w[n]), n
        for p, q in zip(_states(cap), _states(eager)):
            assert torch.equal(p, q)


def _states(m):
    return [s for t in m.opt.list.tensors for s in (t.m, t.v, t.master, t.m_exp, t.v_exp) if s is not None]


def test_moments_of_both_kinds():
    m = Model(torch.bfloat16, bits=8)
    x, a, t = _batch(0, torch.bfloat16)
    m.gradients(x, a, t)
    m.opt.step()
    kinds = set()
    for (mm, vv), tensor in zip(m.opt.moments(), m.opt.list.tensors):
        kinds.add(tensor.m_exp is None)
        g = tensor.g.reshape(-1).double()
        # the first step's: a tenth of the gradient, a twentieth of its square, off by a code (1/8, 1/16)
        # and, of m, by what 16 octaves below a block's largest flush
        assert ((mm.double() - 0.1 * g).abs() <= 0.1 * g.abs() / 8 + 0.1 * g.abs().max() * 2.0 ** -14).all()
        assert ((vv.double() - 0.05 * g * g).abs() <= 0.05 * g * g / 16 + 0.05 * (g * g).max() * 2.0 ** -14).all()
    assert kinds == {True, False}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [T, 7])
def test_serving_step(dtype, n):
    """The norm's rows in 8 bits, handed to the layer, give what the layer makes of tokens that
    quantise to the same integers; fewer tokens than the layer's T among them."""
    g = torch.Generator().manual_seed(5)
    r = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dev()).to(dtype)
    x, a, gw = r(n, d), r(n, d), 1 + r(d, std=0.1)
    experts = QuantizedExperts(r(E, f, d, std=0.15), r(E, f, d, std=0.15), r(E, d, f, std=0.15))
    norm = RMSNorm(T, d, dtype, EPS, quantized=True)
    L = MoELayer(T, d, E, k, f, "swiglu", dtype, rows_alloc_for("exact", T, k, E))
    w_g = r(E, d, std=0.3)
    y = norm.forward(x, gw, add=a)
    q, scale = norm.quantized(n)
    out = L.forward_i8(y, experts, w_g=w_g, renorm=1, quantized=(q, scale)).clone()
    ids, weights = L.ids[:n].clone(), L.weights[:n].clone()
    # by hand: the int8 FFN on the dispatched integers, expert by expert
    want = torch.zeros(n, d, dtype=torch.float64)
    qd, sd = q[:, :d].double().cpu(), scale.double().cpu()
    up = lambda w, s, e: (qd @ w[e, :, :d].double().cpu().T) * sd[:, None] * s[e].double().cpu()
    worst = torch.zeros(n, 1, dtype=torch.float64)
    for e in range(E):
        h = torch.nn.functional.silu(up(experts.w1, experts.s1, e)) * up(experts.w3, experts.s3, e)
        w2 = experts.w2[e, :, :f].double().cpu() * experts.s2[e].double().cpu()[:, None]
        c = (weights.double().cpu() * (ids.cpu() == e)).sum(1, keepdim=True)
        want += c * (h @ w2.T)
        # A as the layer dtype and 8 bits: half a step of each of its row's largest
        step = h.abs().amax(1, keepdim=True) * (1 / 254 + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -20))
        worst += c * step * w2.abs().sum(1).max()
    got = out.double().cpu()
    assert ((got - want).abs() <= worst + 2.0 ** -7 * want.abs() * (dtype == torch.bfloat16) + 1e-5).all()
    # the same integers through the layer's own quantisation
    if dtype == torch.float32:
        again = L.forward_i8(q[:, :d].float() * scale[:, None], experts, ids=ids, weights=weights)
        assert torch.equal(L.xq[:n], q)
        assert (again - out).abs().max() <= 1e-5 * out.abs().max()


def test_serving_refuses_other_rows():
    L = MoELayer(T, d, E, k, f, "swiglu", torch.float32, rows_alloc_for("exact", T, k, E))
    experts = QuantizedExperts(*(torch.zeros(E, *s, device=dev()) for s in ((f, d), (f, d), (d, f))))
    x, w_g = torch.zeros(9, d, device=dev()), torch.zeros(E, d, device=dev())
    q, s = torch.zeros(9, d, dtype=torch.int8, device=dev()), torch.zeros(9, device=dev())
    L.forward_i8(x, experts, w_g=w_g, quantized=(q, s))
    for bad in ((q[:8], s), (q, s[:8]), (q.float(), s), (q, s.double()), (q[:, :48], s), (torch.zeros(9, 2 * d, dtype=torch.int8,
                device=dev())[:, :d], s)):
        with pytest.raises(ValueError):
            L.forward_i8(x, experts, w_g=w_g, quantized=bad)


def test_streams_of_their_own():
    """Two models on two streams at once, each with its own workspaces, leave what they leave alone."""
    x, a, t = _batch(3, torch.bfloat16)
    alone = Model(torch.bfloat16, 8)
    alone.opt.prepare()
    alone.step(x, a, t)
    torch.cuda.synchronize()
    both = [Model(torch.bfloat16, 8) for _ in "12"]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for m, s in zip(both, streams):
        with torch.cuda.stream(s):
            m.opt.prepare()
            m.step(x, a, t)
    torch.cuda.synchronize()
    for m in both:
        for n in m.names:
            assert torch.equal(m.w[n], alone.w[n]), n
