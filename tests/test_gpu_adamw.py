"""The AdamW step on the GPU against the oracle: 32-bit states and weights within the
roundings of float32, 8-bit states code for code.

U = 2^-24.  32-bit: m and v are sums of two rounded products (4 U of their terms'
sizes).  p: the update is lr c1 m / (sqrt(v) c2 + eps), with m and v as above, three
rounded constants, root, quotient and products: 16 U of it, and 2 U of p."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import dev, to_np
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f32": U}
HYPER = dict(lr=0.01, beta1=0.9, beta2=0.99, eps=1e-7, step=7)


def _wrap(a, dtype=torch.float32):
    """a on the device with 16 more elements behind it that must not change."""
    t = torch.full((len(a) + 16,), 77, dtype=dtype, device=dev())
    t[:len(a)] = torch.from_numpy(np.ascontiguousarray(a)).to(dev()).to(dtype)
    return t


class Case:
    """A tensor of n values with the oracle's view of it."""

    def __init__(self, n, rng, bits, p="f32", g="f32", master=False, decay=0.0, place=0):
        self.n, self.bits, self.p_dt, self.place, self.decay = n, bits, p, place, decay
        size = np.exp(rng.uniform(-9, 0, n))
        grad = rng.standard_normal(n) * size
        m, v = (grad * 0.5 + size * 0.1), np.square(size) * rng.uniform(0.1, 3, n)
        w = rng.standard_normal(n).astype(np.float32)
        self.wide = dict(p=_wrap(w, DT[p]), g=_wrap(grad.astype(np.float32), DT[g]))
        if master:
            self.wide["master"] = _wrap(w)
        zero = np.zeros(n, np.int64)
        if bits == 8:
            (cm, em), (cv, ev) = O.adamw_encode(m, zero, 3), O.adamw_encode(v, zero, 4)
            self.wide.update({k: _wrap(a, torch.uint8) for k, a in dict(m=cm, v=cv, m_exp=em, v_exp=ev).items()})
        else:
            self.wide.update(m=_wrap(m.astype(np.float32)), v=_wrap(v.astype(np.float32)))
        self.len = {k: -(-n // 128) if k.endswith("exp") else n for k in self.wide}

    def __getitem__(self, k):
        return self.wide[k][:self.len[k]]

    def tensor(self):
        return B.AdamWTensor(**{k: self[k] for k in self.wide}, weight_decay=self.decay)

    def host(self):
        return {k: to_np(self[k].float()) if k in ("p", "g", "master") or self.bits == 32 else self[k].cpu().numpy()
                for k in self.wide}

    def check(self, before, scale=1.0, seed=0, hyper=HYPER):
        """Against the oracle's step from `before`."""
        now, h = self.host(), hyper
        g = before["g"] * scale
        m0, v0 = before["m"], before["v"]
        if self.bits == 8:
            m0, v0 = O.adamw_decode(m0, before["m_exp"], 3), O.adamw_decode(v0, before["v_exp"], 4)
        p0 = before.get("master", before["p"])
        p, m, v = O.adamw(p0, g, m0, v0, h["lr"], h["beta1"], h["beta2"], h["eps"], h["step"], self.decay)
        me = 4 * U * (np.abs(h["beta1"] * m0) + (1 - h["beta1"]) * np.abs(g))
        if self.bits == 8:
            rm, rv = O.adamw_random(self.n, seed, self.place)
            for k, x, r, mant in (("m", m, rm, 3), ("v", v, rv, 4)):
                c, e = O.adamw_encode(x, r, mant)
                np.testing.assert_array_equal(now[k], c)
                np.testing.assert_array_equal(now[k + "_exp"], e)
        else:
            assert (np.abs(now["m"] - m) <= me).all() and (np.abs(now["v"] - v) <= 4 * U * v).all()
        c1, c2 = 1 / (1 - h["beta1"] ** h["step"]), (1 - h["beta2"] ** h["step"]) ** -0.5
        den = np.sqrt(v) * c2 + h["eps"]
        bound = h["lr"] * c1 / den * (16 * U * np.abs(m) + me) + 2 * U * (np.abs(p) + np.abs(p0))
        if "master" in now:
            assert (np.abs(now["master"] - p) <= bound).all()
            assert torch.equal(self["p"], self["master"].to(DT[self.p_dt]))
        else:
            assert (np.abs(now["p"] - p) <= bound + ROUND[self.p_dt] * np.abs(p)).all()
        np.testing.assert_array_equal(now["g"], before["g"])
        for k, t in self.wide.items():
            assert (t[self.len[k]:] == 77).all(), k


KINDS = [dict(bits=32), dict(bits=32, g="bf16"), dict(bits=32, p="bf16"), dict(bits=32, p="bf16", master=True),
         dict(bits=8), dict(bits=8, p="bf16"), dict(bits=8, p="bf16", master=True), dict(bits=8, p="bf16", g="bf16")]


@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_one_tensor(kind):
    for n in (1, 7, 8, 127, 128, 129, 1000, 2048, 2051, 8192, 70001):
        c = Case(n, np.random.default_rng(n), decay=0.1, **kind)
        before = c.host()
        B.moe_adamw(B.AdamWList([c.tensor()]), **HYPER, seed=n)
        c.check(before, seed=n)


@pytest.mark.parametrize("count", [2, 40, 41, 90])
def test_many_tensors(count):
    """Lists around a launch's 40 tensors, of every kind and odd sizes, empty ones among them; a scale on
    the device."""
    rng = np.random.default_rng(count)
    cases = [Case(int(rng.choice([0, 1, 5, 64, 300, 4099])), rng, place=i, decay=float(i % 3) / 10, **KINDS[i % len(KINDS)])
             for i in range(count)]
    before = [c.host() for c in cases]
    scale = torch.tensor([0.25], device=dev())
    B.moe_adamw(B.AdamWList([c.tensor() for c in cases]), **HYPER, seed=0xF0000005, grad_scale=scale)
    for c, b in zip(cases, before):
        c.check(b, scale=0.25, seed=0xF0000005)


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[6]], ids=str)
def test_a_large_tensor_takes_chunks_of_more_tiles(kind):
    n = 40_000_003
    rng = np.random.default_rng(1)
    c = Case(n, rng, **kind)
    before = c.host()
    B.moe_adamw(B.AdamWList([c.tensor()]), **HYPER, seed=3)
    c.check(before, seed=3)


def test_unpack():
    cases = [Case(n, np.random.default_rng(n), bits=8, place=i) for i, n in enumerate((5, 128, 1000, 70001))]
    values = [[torch.full((c.n + 4,), 7.0, device=dev()) for _ in "mv"] for c in cases]
    B.moe_adamw_unpack(B.AdamWList([c.tensor() for c in cases]), values)
    for c, (m, v) in zip(cases, values):
        h = c.host()
        np.testing.assert_array_equal(to_np(m[:c.n]), O.adamw_decode(h["m"], h["m_exp"], 3))
        np.testing.assert_array_equal(to_np(v[:c.n]), O.adamw_decode(h["v"], h["v_exp"], 4))
        assert (m[c.n:] == 7).all() and (v[c.n:] == 7).all()


def test_from_zero_states():
    """The first step, from states of zeros: m and v are the gradient's, p moves by lr."""
    n = 300
    g = torch.randn(n, generator=torch.Generator().manual_seed(0)).to(dev())
    g[5] = 0
    z8 = lambda k: torch.zeros(k, dtype=torch.uint8, device=dev())
    p = torch.zeros(n, device=dev())
    t = B.AdamWTensor(p, g, z8(n), z8(n), m_exp=z8(3), v_exp=z8(3))
    B.moe_adamw(B.AdamWList([t]), 0.01, 0.9, 0.99, 1e-12, 1)
    assert p[5] == 0 and t.m[5] == 0 and t.v[5] == 0
    live = torch.arange(n, device=dev()) != 5
    assert torch.allclose(p[live], -0.01 * g[live].sign(), rtol=1e-5)
    z8 = torch.zeros(n, device=dev())
    q = torch.zeros(n, device=dev())
    B.moe_adamw(B.AdamWList([B.AdamWTensor(q, g, z8, z8.clone())]), 0.01, 0.9, 0.99, 1e-12, 1)
    assert torch.allclose(p, q, rtol=1e-5, atol=0)


@pytest.mark.parametrize("bits", [8, 32])
def test_least_eps(bits):
    """v = 0 leaves eps alone to divide by: 0 / eps is 0 for the least eps that is taken."""
    n, eps = 300, 2.0 ** -126
    zero = lambda k, t=torch.float32: torch.zeros(k, dtype=t, device=dev())
    u8 = torch.uint8
    m, v, e = (zero(n, u8), zero(n, u8), dict(m_exp=zero(3, u8), v_exp=zero(3, u8))) if bits == 8 else (zero(n), zero(n), {})
    p, g = torch.ones(n, device=dev()), zero(n)
    B.moe_adamw(B.AdamWList([B.AdamWTensor(p, g, m, v, **e)]), 0.01, 0.9, 0.99, eps, 1)
    assert (p == 1).all() and not m.any() and not v.any()


@pytest.mark.parametrize("bits", [8, 32])
def test_gradients_that_are_not_finite_stay_in_their_element(bits):
    n, rng = 256, np.random.default_rng(0)
    c = Case(n, rng, bits)
    ref = Case(n, np.random.default_rng(0), bits)
    for at, x in ((3, np.nan), (50, np.inf), (51, -np.inf), (130, 3e38)):
        c["g"][at] = x
    for t in (c, ref):
        B.moe_adamw(B.AdamWList([t.tensor()]), **HYPER)
    odd = np.zeros(n, bool)
    odd[[3, 50, 51, 130]] = True
    got, want = c.host(), ref.host()
    assert np.isnan(got["p"][odd][:3]).all() and np.isfinite(got["p"][130])
    np.testing.assert_array_equal(got["p"][~odd], want["p"][~odd])
    if bits == 8:
        assert (got["m"][[3, 50, 51]] == 128).all() and (got["v"][odd] == 255).all()
        # (the second block's exponent of m is that of its finite 3e37)
        np.testing.assert_array_equal(got["m"][:128][~odd[:128]], want["m"][:128][~odd[:128]])
        np.testing.assert_array_equal(got["v"][~odd], want["v"][~odd])
    else:
        np.testing.assert_array_equal(got["m"][~odd], want["m"][~odd])
    # and so they stay
    for at in (3, 50, 51, 130):
        c["g"][at] = 1.0
    B.moe_adamw(B.AdamWList([c.tensor()]), **HYPER)
    assert np.isnan(c.host()["p"][odd][:3]).all() and np.isfinite(c.host()["p"][~odd]).all()


def test_states_in_8_bits_follow_those_in_32():
    """400 steps of beta2 = 0.999 with gradients whose size falls: rounded to nearest, v would stay
    where it began.  Of its mean over 4096 elements: a step adds an error of mean 0 and a standard
    deviation of at most half a code, 1/32 of v, so 400 of them sqrt(400) / 32 = 0.63 an element and
    1 % of the mean; five of those."""
    n, gen = 4096, torch.Generator().manual_seed(1)
    mk = lambda k, dtype: torch.zeros(k, dtype=dtype, device=dev())
    p8, p32, g = mk(n, torch.float32), mk(n, torch.float32), mk(n, torch.float32)
    a = B.AdamWTensor(p8, g, mk(n, torch.uint8), mk(n, torch.uint8), m_exp=mk(32, torch.uint8), v_exp=mk(32, torch.uint8))
    b = B.AdamWTensor(p32, g, mk(n, torch.float32), mk(n, torch.float32))
    both, out = B.AdamWList([a, b]), [[mk(n, torch.float32), mk(n, torch.float32)]]
    for step in range(1, 401):
        g.copy_(torch.randn(n, generator=gen) * (1.0 if step <= 100 else 0.1))
        B.moe_adamw(both, 1e-3, 0.9, 0.999, 1e-8, step, seed=step)
    B.moe_adamw_unpack(B.AdamWList([a]), out)
    v8, v32 = out[0][1].double().mean().item(), b.v.double().mean().item()
    assert abs(v8 / v32 - 1) < 0.05
    assert v32 < 0.08                            # (it has come down from 0.095)


def test_captured_steps_take_their_schedule_from_the_device():
    """Replays with other gradients and schedules equal eager steps with the same numbers."""
    kinds = [KINDS[0], KINDS[6], KINDS[3]]
    cases = [[Case(5000 + i, np.random.default_rng(i), place=i, decay=0.1, **k) for i, k in enumerate(kinds)] for _ in range(2)]
    lists = [B.AdamWList([c.tensor() for c in cs]) for cs in cases]
    schedule, scale = torch.zeros(4, device=dev()), torch.ones(1, device=dev())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.moe_adamw(lists[0], 0.0, 0.9, 0.99, 1e-8, 1, grad_scale=scale, schedule=schedule)
    for step in range(1, 5):
        gen = torch.Generator().manual_seed(step)
        for a, b in zip(*cases):
            g = torch.randn(a.n, generator=gen).to(dev())
            a["g"].copy_(g)
            b["g"].copy_(g)
        lr, seed = 0.01 / step, 0xFFFFFFF0 + step
        schedule.copy_(B.adamw_schedule(lr, 0.9, 0.99, step, seed))
        scale.fill_(1.0 / step)
        graph.replay()
        B.moe_adamw(lists[1], lr, 0.9, 0.99, 1e-8, step, seed=seed, grad_scale=scale)
        torch.cuda.synchronize()
        for a, b in zip(*cases):
            for k in a.wide:
                assert torch.equal(a.wide[k], b.wide[k]), (step, k)


def test_elements_past_32_bits():
    """A tensor of more than 2^32 values: its parts around 2^31 and 2^32 and its end, codes and all."""
    n = (1 << 32) + 300
    g = torch.Generator(device="cuda").manual_seed(0)
    u8 = lambda k: torch.zeros(k, dtype=torch.uint8, device=dev())
    p, grad = torch.zeros(n, dtype=torch.bfloat16, device=dev()), torch.zeros(n, dtype=torch.bfloat16, device=dev())
    parts = [slice(0, 1024), slice((1 << 31) - 512, (1 << 31) + 512), slice((1 << 32) - 512, n - 300 + 256), slice(n - 300 + 256, n)]
    for s in parts:
        grad[s] = torch.randn(s.stop - s.start, generator=g, device="cuda").to(torch.bfloat16)
    t = B.AdamWTensor(p, grad, u8(n), u8(n), m_exp=u8(B.adamw_blocks(n)), v_exp=u8(B.adamw_blocks(n)))
    B.moe_adamw(B.AdamWList([t]), **HYPER, seed=9)
    for s in parts:
        k, blocks = s.stop - s.start, slice(s.start // 128, -(-s.stop // 128))
        gr = to_np(grad[s])
        _, m, v = O.adamw(np.zeros(k), gr, np.zeros(k), np.zeros(k), 0.01, 0.9, 0.99, 1e-7, 7)
        rm, rv = O.adamw_random(k, 9, 0, start=s.start)
        for x, r, mant, code, e in ((m, rm, 3, t.m, t.m_exp), (v, rv, 4, t.v, t.v_exp)):
            c, ee = O.adamw_encode(x, r, mant)
            np.testing.assert_array_equal(code[s].cpu().numpy(), c)
            np.testing.assert_array_equal(e[blocks].cpu().numpy(), ee)
        assert (p[s][grad[s] != 0] != 0).all()
