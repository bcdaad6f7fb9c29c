"""The root-mean-square norm on the GPU against the oracle: forward with and
without the addition, rows in 8 bits (every integer equal), backward.

Tolerances: U = 2^-24 a rounding of float32, ROUND one of the result to its type.
A row's squares are added by at most 32 additions in a thread, 6 in a wavefront
and 16 between wavefronts, so mean, root and quotient leave r within 32 U."""
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
EPS = 1e-5
R_ERR = 32 * U


def _wide(rows, d, pad, dt, rng, scale=1.0, fill=7.0):
    """[rows, d] cut out of a buffer with pad columns and a row behind it."""
    t = torch.full((rows + 1, d + pad), fill, dtype=DT[dt], device=dev())
    v = rng.standard_normal((rows, d)) * rng.uniform(0.2, 5, (rows, 1)) * scale
    t[:rows, :d] = torch.from_numpy(v.astype(np.float32)).to(dev()).to(DT[dt])
    return t, t[:rows, :d]


def _untouched(wide, rows, d, fill=7.0):
    assert (wide[rows:] == fill).all() and (wide[:rows, d:] == fill).all()


def near(got, ref, bound):
    err = np.abs(to_np(got) - ref) - bound
    i = int(np.argmax(err))
    assert (err <= 0).all(), (i, to_np(got).flat[i], ref.flat[i], bound.flat[i] if bound.ndim else bound)


SIZES = [(1, 8, 0), (3, 24, 8), (5, 512, 0), (40, 520, 8), (130, 1000, 24), (9, 2048, 0), (7, 2056, 0), (1, 4096, 0),
         (300, 4096, 8), (11, 8192, 0), (4, 8200, 40), (3, 16384, 0), (2, 16392, 0), (2, 32768, 8)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,pad", SIZES)
@pytest.mark.parametrize("add", [False, True])
def test_forward(dt, rows, d, pad, add):
    rng = np.random.default_rng(rows * d + pad)
    _, x = _wide(rows, d, pad, dt, rng)
    _, a = _wide(rows, d, pad, dt, rng, 3.0)
    w = torch.from_numpy(rng.uniform(-1.5, 1.5, d).astype(np.float32)).to(dev()).to(DT[dt])
    sw, s = _wide(rows, d, pad, dt, rng)
    yw, y = _wide(rows, d, pad, dt, rng)
    rstd = torch.full((rows + 1,), 5.0, device=dev())
    q = torch.full((rows + 1, B.quantized_width(d)), 99, dtype=torch.int8, device=dev())
    scale = torch.full((rows + 1,), 5.0, device=dev())
    B.moe_rms_norm_fwd(x, w, EPS, y=y, add=a if add else None, sum=s if add else None, rstd=rstd, q=q, scale=scale)
    torch.cuda.synchronize()
    rs, rr, ry = O.rms_norm_fwd(to_np(x), to_np(w), EPS, to_np(a) if add else None, dt)
    if add:
        np.testing.assert_array_equal(to_np(s), rs)
        _untouched(sw, rows, d)
    near(rstd[:rows], rr, R_ERR * rr)
    near(y, ry, ROUND[dt] * np.abs(ry) + (R_ERR + 3 * U) * np.abs(ry))
    _untouched(yw, rows, d)
    rq, rc = O.rms_norm_rows_i8(rs, rr, to_np(w))
    np.testing.assert_array_equal(q.cpu().numpy()[:rows, :d], rq)
    assert not q[:rows, d:].any() and (q[rows:] == 99).all()
    near(scale[:rows], rc, (R_ERR + 2 * U) * rc)
    assert rstd[rows] == 5 and scale[rows] == 5
    # y alone, q alone and the sum left out give the same bits
    y2, q2, sc2 = torch.empty_like(y), torch.empty_like(q), torch.empty_like(scale)
    B.moe_rms_norm_fwd(x, w, EPS, y=y2, add=a if add else None)
    B.moe_rms_norm_fwd(x, w, EPS, q=q2, scale=sc2, add=a if add else None)
    assert torch.equal(y2, y) and torch.equal(q2[:rows], q[:rows]) and torch.equal(sc2[:rows], scale[:rows])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 4096])
def test_special_rows(dt, d):
    """Zeros, values whose squares vanish or overflow, NaN and infinities: each row by itself."""
    n = np.arange(d)
    rows = [np.zeros(d), np.full(d, 1e-30), np.full(d, 1e25), np.where(n == d // 2, np.nan, 1.0),
            np.where(n == d - 1, np.inf, 2.0), np.where(n == 0, -np.inf, -3.0), np.where(n == 3, 100.0, 0.0),
            np.ones(d)]
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).to(dev()).to(DT[dt])
    w = torch.full((d,), 0.5, dtype=DT[dt], device=dev())
    y, q = torch.empty_like(x), torch.empty(8, B.quantized_width(d), dtype=torch.int8, device=dev())
    scale = torch.empty(8, device=dev())
    B.moe_rms_norm_fwd(x, w, EPS, y=y, q=q, scale=scale)
    y, q, scale = to_np(y), q.cpu().numpy(), scale.cpu().numpy()
    assert not y[0].any() and not q[0].any() and scale[0] == 0
    tiny = to_np(x)[1] * 0.5 / np.sqrt(EPS)
    np.testing.assert_allclose(y[1], tiny, rtol=2.0 ** -7)
    assert (q[1] == 127).all()
    assert not y[2].any() and scale[2] == 0                    # the squares are beyond float32: r = 0
    assert np.isnan(y[3]).all() and np.isnan(scale[3]) and not q[3].any()
    for r, at in ((4, d - 1), (5, 0)):                         # r = 0: infinity times 0, and zeros
        assert np.isnan(y[r][at]) and not np.delete(y[r], at).any()
        assert np.isnan(scale[r]) and not q[r].any()
    ref = 0.5 * 100 / np.sqrt(1e4 / d + EPS)
    assert abs(y[6][3] - ref) <= (2.0 ** -8 + 1e-5) * ref and q[6][3] == 127 and np.count_nonzero(y[6]) == 1
    assert (q[7] == 127).all()


@pytest.mark.parametrize("dt,dw_dt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,d,pad", SIZES + [(2050, 264, 0), (4099, 2056, 8)])
@pytest.mark.parametrize("beside", [False, True])
def test_backward(dt, dw_dt, rows, d, pad, beside):
    rng = np.random.default_rng(rows + d + pad)
    _, s = _wide(rows, d, pad, dt, rng, 2.0)
    _, dy = _wide(rows, d, pad, dt, rng, 0.1)
    _, dsum = _wide(rows, d, pad, dt, rng)
    w = torch.from_numpy(rng.uniform(-1.5, 1.5, d).astype(np.float32)).to(dev()).to(DT[dt])
    S, DY, W, DS = to_np(s), to_np(dy), to_np(w), to_np(dsum) if beside else None
    _, r, _ = O.rms_norm_fwd(S, W, EPS)
    rstd = torch.from_numpy(r.astype(np.float32)).to(dev())
    xw, dx = _wide(rows, d, pad, dt, rng)
    dw = torch.full((d + 8,), 5.0, dtype=DT[dw_dt], device=dev())
    ws = torch.full((B.moe_rms_norm_bwd_workspace_bytes(rows, d) + 64,), 77, dtype=torch.uint8, device=dev())
    B.moe_rms_norm_bwd(s, w, rstd, dy, dx, dw, ws, dsum=dsum if beside else None)
    torch.cuda.synchronize()
    rdx, rdw = O.rms_norm_bwd(S, r, W, DY, DS)
    # r: one rounding; g one, c by at most 64 additions of rounded products, then r (g - s c) + dsum
    g = np.abs(DY * W)
    c = (r * r * (g * np.abs(S)).mean(axis=1))[:, None]
    bound = ROUND[dt] * np.abs(rdx) + U * (8 * r[:, None] * g + 80 * r[:, None] * np.abs(S) * c + 2 * np.abs(rdx))
    near(dx, rdx, bound)
    _untouched(xw, rows, d)
    # additions: a wavefront's rows, its workgroup's, a share of the workgroups', the shares'
    ops = rows / 512 + 4 + 512 / 16 + 16 + 4
    near(dw[:d], rdw, ROUND[dw_dt] * np.abs(rdw) + U * ops * np.abs(DY * S * r[:, None]).sum(axis=0))
    assert (dw[d:] == 5).all() and (ws[-64:] == 77).all()
    # without dw; in place of dy, of s and of dsum
    alone = torch.empty_like(dx)
    B.moe_rms_norm_bwd(s, w, rstd, dy, alone, None, None, dsum=dsum if beside else None)
    assert torch.equal(alone, dx)
    for name in ("dy", "s") + (("dsum",) if beside else ()):
        t = dict(s=s.clone(), dy=dy.clone(), dsum=dsum.clone())
        dw2 = torch.empty_like(dw)
        B.moe_rms_norm_bwd(t["s"], w, rstd, t["dy"], t[name], dw2, ws, dsum=t["dsum"] if beside else None)
        assert torch.equal(t[name], dx) and torch.equal(dw2[:d], dw[:d]), name


def test_backward_is_the_forwards_differences():
    """Central differences of <dy, y> + <dsum, s> in the kernel's own float32 forward."""
    rows, d, h = 3, 40, 1e-2
    g = torch.Generator().manual_seed(3)
    x, a, dy, ds = (torch.randn(rows, d, generator=g).to(dev()) for _ in range(4))
    w = torch.rand(d, generator=g).to(dev()) + 0.5

    def f(x, w):
        s, y = torch.empty_like(x), torch.empty_like(x)
        B.moe_rms_norm_fwd(x, w, EPS, y=y, add=a, sum=s)
        return ((y * dy).double().sum() + (s * ds).double().sum()).item()

    s, y, dx, dw, rstd = (torch.empty_like(t) for t in (x, x, x, w, x[:, 0].contiguous()))
    B.moe_rms_norm_fwd(x, w, EPS, y=y, add=a, sum=s, rstd=rstd)
    B.moe_rms_norm_bwd(s, w, rstd, dy, dx, dw, B.workspace(B.moe_rms_norm_bwd_workspace_bytes(rows, d), dev()), dsum=ds)
    # truncation of order h^2 = 1e-4, roundings of 120 values of about 3: 1e-5 / h
    for i in range(0, rows * d, 7):
        e = torch.zeros(rows * d, device=dev())
        e[i] = h
        e = e.view(rows, d)
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx.view(-1)[i].item()) < 5e-3
    for j in range(d):
        e = torch.zeros(d, device=dev())
        e[j] = h
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[j].item()) < 5e-3


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [256, 4096, 9000])
def test_in_place(dt, d):
    """sum over x or add, y over the other."""
    rng = np.random.default_rng(d)
    x, a = (_wide(33, d, 0, dt, rng)[1] for _ in range(2))
    w = torch.ones(d, dtype=DT[dt], device=dev())
    s, y = torch.empty_like(x), torch.empty_like(x)
    B.moe_rms_norm_fwd(x, w, EPS, y=y, add=a, sum=s)
    for swap in (False, True):
        x2, a2 = x.clone(), a.clone()
        B.moe_rms_norm_fwd(x2, w, EPS, y=a2 if swap else x2, add=a2, sum=x2 if swap else a2)
        assert torch.equal(x2 if swap else a2, s) and torch.equal(a2 if swap else x2, y)


def test_no_rows():
    w = torch.ones(16, device=dev())
    e = torch.empty(0, 16, device=dev())
    B.moe_rms_norm_fwd(e, w, EPS, y=torch.empty_like(e))
    dw = torch.full((16,), 5.0, device=dev())
    B.moe_rms_norm_bwd(e, w, torch.empty(0, device=dev()), e, torch.empty_like(e), dw, B.workspace(0, dev()))
    assert not dw.any()


def test_rows_past_32_bit_offsets():
    """Rows 2^29 elements apart, so that the last ones lie past 2^31 elements."""
    d, ld, rows = 64, 1 << 29, 6
    big = torch.empty((rows - 1) * ld + d, dtype=torch.bfloat16, device=dev())
    x = big.as_strided((rows, d), (ld, 1))
    x.copy_(torch.randn(rows, d, device=dev()))
    w = torch.ones(d, dtype=torch.bfloat16, device=dev())
    y, ref = torch.empty(rows, d, dtype=torch.bfloat16, device=dev()), torch.empty(rows, d, dtype=torch.bfloat16, device=dev())
    B.moe_rms_norm_fwd(x, w, EPS, y=y)
    B.moe_rms_norm_fwd(x.contiguous(), w, EPS, y=ref)
    assert torch.equal(y, ref)
    B.moe_rms_norm_fwd(ref, w, EPS, y=x)
    B.moe_rms_norm_fwd(ref, w, EPS, y=y)
    assert torch.equal(x.contiguous(), y)


def test_captured_and_replayed():
    """Forward and backward in one graph, replayed on other inputs beside eager work."""
    rows, d = 515, 4096
    g = torch.Generator().manual_seed(0)
    new = lambda *s: torch.randn(*s, generator=g).to(dev()).to(torch.bfloat16)
    x, a, dy, w = new(rows, d), new(rows, d), new(rows, d), new(d)
    ws = B.workspace(B.moe_rms_norm_bwd_workspace_bytes(rows, d), dev())
    out = lambda: dict(s=torch.empty_like(x), y=torch.empty_like(x), dx=torch.empty_like(x), dw=torch.empty(d, device=dev()),
                       r=torch.empty(rows, device=dev()), c=torch.empty(rows, device=dev()),
                       q=torch.empty(rows, d, dtype=torch.int8, device=dev()))

    def step(o, ws):
        B.moe_rms_norm_fwd(x, w, EPS, y=o["y"], add=a, sum=o["s"], rstd=o["r"], q=o["q"], scale=o["c"])
        B.moe_rms_norm_bwd(o["s"], w, o["r"], dy, o["dx"], o["dw"], ws)

    o, e = out(), out()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(o, ws)
    for _ in range(4):
        for t in (x, a, dy):
            t.copy_(new(*t.shape))
        graph.replay()
        step(e, torch.empty_like(ws))
        torch.cuda.synchronize()
        for n in o:
            assert torch.equal(o[n], e[n]), n
