"""What the operators around the layer refuse, on the CPU: the binding before any
device access, the C entry points before any launch."""
import ctypes
import math

import pytest
import torch

from paper_2205_01848_amd import binding as B

bf16, f32, i32, i8, u8 = torch.bfloat16, torch.float32, torch.int32, torch.int8, torch.uint8
EINVAL, EWORKSPACE = 1, 4


def z(*s, dt=f32):
    return torch.zeros(*s, dtype=dt)


def passes_checks(fn, **kw):
    """fn(**kw) gets past the size and type checks: it fails only for want of a device."""
    with pytest.raises((B.MoEError, RuntimeError)) as e:
        fn(**kw)
    assert "device memory" in str(e.value) or "GPU" in str(e.value), e.value


def refuses(match, fn, **kw):
    with pytest.raises(B.MoEError, match=match):
        fn(**kw)


NORM = dict(x=z(5, 24), weight=z(24), eps=1e-5, y=z(5, 24), add=z(5, 24), sum=z(5, 24), rstd=z(5),
            q=z(5, 32, dt=i8), scale=z(5))
NORM_BWD = dict(s=z(5, 24), weight=z(24), rstd=z(5), dy=z(5, 24), dx=z(5, 24), dw=z(24), ws=z(4096, dt=u8),
                dsum=z(5, 24))
LOSS = dict(x=z(5, 24), w=z(7, 24), targets=z(5, dt=i32), loss=z(5), lse=z(5), status=z(1, dt=i32),
            ws=z(1 << 16, dt=u8), weights=z(5), dx=z(5, 24), dw=z(7, 24))
CALLS = [(B.moe_rms_norm_fwd, NORM, "x"), (B.moe_rms_norm_bwd, NORM_BWD, "s"), (B.moe_vocab_loss, LOSS, "x")]
OPERANDS = [(fn, kw, n) for fn, kw, first in CALLS for n, t in kw.items()
            if torch.is_tensor(t) and n not in ("ws", first)]


@pytest.mark.parametrize("fn,kw", [c[:2] for c in CALLS], ids=lambda v: getattr(v, "__name__", ""))
def test_sizes_that_fit_reach_the_device_check(fn, kw):
    passes_checks(fn, **kw)


@pytest.mark.parametrize("fn,kw,name", OPERANDS)
def test_every_operand_too_small_or_of_another_type(fn, kw, name):
    t = kw[name]
    if fn is not B.moe_vocab_loss or name != "w":     # (fewer words are another vocabulary)
        refuses(name, fn, **dict(kw, **{name: t[:-1].contiguous()}))
    refuses(name, fn, **dict(kw, **{name: t.to(torch.float64)}))


@pytest.mark.parametrize("fn,kw,name", [o for o in OPERANDS if o[1][o[2]].dim() == 2 and o[2] != "q" and o[1] is not LOSS or o[2] == "dx"])
def test_rows_with_gaps(fn, kw, name):
    passes_checks(fn, **dict(kw, **{name: z(5, 32)[:, :24]}))
    refuses(name, fn, **dict(kw, **{name: z(5, 28)[:, :24]}))          # 28 elements apart
    refuses(name, fn, **dict(kw, **{name: z(24, 5).T}))


P = ctypes.c_void_p(4096)       # an aligned address that is never read


def _norm(lib, dt=1, rows=5, d=24, x=P, ldx=24, add=P, ldadd=24, w=P, eps=1e-5, sum=ctypes.c_void_p(8192), ldsum=24,
          y=P, ldy=24, rstd=None, q=None, scale=None):
    return lib.moe_rms_norm_fwd(None, dt, rows, d, x, ldx, add, ldadd, w, eps, sum, ldsum, y, ldy, rstd, q, scale)


@pytest.mark.parametrize("kw", [
    dict(dt=2), dict(rows=-1), dict(d=0), dict(d=20), dict(d=32776, ldx=32776, ldadd=32776, ldsum=32776, ldy=32776),
    dict(x=None), dict(w=None), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan),
    dict(ldx=16), dict(ldx=28), dict(ldadd=20), dict(ldsum=16), dict(ldy=23), dict(y=None), dict(q=P), dict(scale=P),
    dict(add=None), dict(sum=P), dict(x=ctypes.c_void_p(4100)), dict(y=ctypes.c_void_p(4104)),
    dict(q=ctypes.c_void_p(4097), scale=P), dict(w=ctypes.c_void_p(4098)),
    # over an input whose rows lie otherwise
    dict(add=ctypes.c_void_p(12288), ldy=32), dict(x=ctypes.c_void_p(12288), ldadd=32),
    dict(y=ctypes.c_void_p(12288), sum=P, ldsum=32), dict(add=ctypes.c_void_p(8192), ldsum=32, y=None, q=P, scale=P)], ids=str)
def test_norm_refuses(kw):
    assert _norm(B.lib(), **kw) == EINVAL


def _norm_bwd(lib, dt=1, rows=5, d=24, s=P, lds=24, w=P, rstd=P, dy=P, lddy=24, dsum=P, lddsum=24, dx=P, lddx=24,
              dw_dt=1, dw=P, ws=P, nws=1 << 20):
    return lib.moe_rms_norm_bwd(None, dt, rows, d, s, lds, w, rstd, dy, lddy, dsum, lddsum, dx, lddx, dw_dt, dw, ws, nws)


@pytest.mark.parametrize("kw,st", [
    (dict(dt=3), EINVAL), (dict(rows=-1), EINVAL), (dict(d=12), EINVAL), (dict(s=None), EINVAL), (dict(w=None), EINVAL),
    (dict(rstd=None), EINVAL), (dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(lds=23), EINVAL),
    (dict(lddy=16), EINVAL), (dict(lddsum=25), EINVAL), (dict(lddx=16), EINVAL), (dict(dw_dt=2), EINVAL),
    (dict(dt=0, dw_dt=1), EINVAL), (dict(dx=ctypes.c_void_p(4104)), EINVAL), (dict(ws=None), EWORKSPACE),
    (dict(lddx=32), EINVAL), (dict(dy=ctypes.c_void_p(8192), dsum=None, lds=32), EINVAL),   # dx over rows that lie otherwise
    (dict(s=ctypes.c_void_p(8192), dsum=None, lddy=32), EINVAL),
    (dict(s=ctypes.c_void_p(8192), dy=ctypes.c_void_p(8192), lddsum=32), EINVAL),
    (dict(nws=2 * 24 * 4 - 1), EWORKSPACE), (dict(ws=ctypes.c_void_p(4100)), EWORKSPACE)], ids=str)
def test_norm_bwd_refuses(kw, st):
    assert _norm_bwd(B.lib(), **kw) == st


def test_norm_workspace():
    """One partial sum a workgroup, 512 at most; nothing for sizes the call refuses."""
    q = B.moe_rms_norm_bwd_workspace_bytes
    assert q(0, 24) == q(1, 24) == q(4, 24) == 96 and q(5, 24) == 192 and q(1 << 40, 4096) == 512 * 4096 * 4
    assert q(3, 4096) == 3 * 4096 * 4
    assert q(-1, 24) == q(5, 20) == q(5, 32776) == 0


def _list(n=200, bits=8, master=False, p=bf16, **kw):
    t = dict(p=z(n, dt=p), g=z(n), m=z(n), v=z(n), weight_decay=0.1)
    if bits == 8:
        t.update(m=z(n, dt=u8), v=z(n, dt=u8), m_exp=z(2, dt=u8), v_exp=z(2, dt=u8))
    if master:
        t["master"] = z(n)
    return dict(t, **kw)


@pytest.mark.parametrize("match,kw", [
    ("g holds", dict(g=z(199))), ("g holds", dict(g=z(201))), ("m holds", dict(m=z(199, dt=u8))),
    ("v holds", dict(v=z(201, dt=u8))), ("m_exp holds", dict(m_exp=z(1, dt=u8))), ("v_exp holds", dict(v_exp=z(3, dt=u8))),
    ("v_exp: both", dict(v_exp=None)), ("m: element type", dict(m=z(200))), ("v: element type", dict(v=z(200))),
    ("m: element type", dict(m_exp=None, v_exp=None)), ("master: only", dict(p=z(200), master=z(200))),
    ("master: element", dict(master=z(200, dt=bf16))), ("master holds", dict(master=z(100))),
    ("unsupported", dict(p=z(200, dt=torch.float16))), ("unsupported", dict(g=z(200, dt=torch.float64)))], ids=str)
def test_adamw_tensor_refuses(match, kw):
    B.AdamWTensor(**_list())
    refuses(match, B.AdamWTensor, **dict(_list(), **kw))


def _adamw(lib, count=1, lr=0.1, b1=0.9, b2=0.99, eps=1e-8, step=1, scale=None, schedule=None, tensors=True, **kw):
    a = ctypes.addressof(ctypes.create_string_buffer(16)) // 16 * 16 + 16
    f = dict(p=a, g=a, master=None, m=a, v=a, m_exp=None, v_exp=None, n=0, weight_decay=0.0, p_dtype=1, g_dtype=0)
    f.update(kw)
    arr = (B.AdamWTensorArgs * 1)(B.AdamWTensorArgs(*f.values()))
    return lib.moe_adamw(None, count, arr if tensors else None, lr, b1, b2, eps, step, 0, scale, schedule)


@pytest.mark.parametrize("kw", [
    dict(count=-1), dict(tensors=False), dict(lr=-0.1), dict(lr=math.nan), dict(lr=math.inf), dict(b1=1.0), dict(b1=-0.1),
    dict(b2=1.0), dict(b2=math.nan), dict(eps=0.0), dict(eps=1e-60), dict(eps=1e-40), dict(eps=math.inf), dict(step=0), dict(n=-1),
    dict(p_dtype=2), dict(g_dtype=-1), dict(weight_decay=-1.0), dict(weight_decay=math.nan), dict(m_exp=64), dict(v_exp=64),
    dict(p_dtype=0, master=64), dict(n=5, p=None), dict(n=5, g=None), dict(n=5, m=None), dict(n=5, v=None),
    dict(n=5, p=72), dict(n=5, g=66), dict(n=5, master=68), dict(n=5, m=65), dict(n=5, v=72), dict(n=(1 << 40) + 1),
    dict(scale=66), dict(schedule=65)], ids=str)
def test_adamw_refuses(kw):
    assert _adamw(B.lib()) == 0 and _adamw(B.lib(), **kw) == EINVAL


def test_adamw_of_nothing():
    assert B.lib().moe_adamw(None, 0, None, 0.1, 0.9, 0.99, 1e-8, 1, 0, None, None) == 0
    assert B.lib().moe_adamw_unpack(None, 0, None, None, None) == 0
    assert [B.lib().moe_adamw_blocks(n) for n in (-1, 0, 1, 128, 129)] == [0, 0, 1, 1, 2] == \
        [max(0, B.adamw_blocks(n)) for n in (-1, 0, 1, 128, 129)]


def test_adamw_schedule():
    t = B.adamw_schedule(0.5, 0.5, 0.75, 2, seed=0xFFFFFFFE)
    assert t[:3].tolist() == [0.5, pytest.approx(4 / 3), pytest.approx((1 - 0.5625) ** -0.5)]
    assert t.view(i32)[3] == -2 and B.adamw_schedule(0.5, 0.5, 0.75, 2, seed=5).view(i32)[3] == 5


def test_loss_takes_both_gradients_or_none():
    passes_checks(B.moe_vocab_loss, **dict(LOSS, dx=None, dw=None))
    refuses("both or neither", B.moe_vocab_loss, **dict(LOSS, dx=None))
    refuses("both or neither", B.moe_vocab_loss, **dict(LOSS, dw=None))
    refuses("w has shape", B.moe_vocab_loss, **dict(LOSS, w=z(7, 32)))
    passes_checks(B.moe_vocab_loss, **dict(LOSS, w=z(9, 24), dw=z(9, 24)))


def _loss(lib, dt=1, T=5, d=24, V=7, x=P, ldx=24, w=P, targets=P, scale=1.0, weights=None, loss=P, lse=None, dx=P,
          lddx=24, dw_dt=1, dw=P, status=P, ws=P, nws=1 << 30):
    return lib.moe_vocab_loss(None, dt, T, d, V, x, ldx, w, targets, scale, weights, loss, lse, dx, lddx, dw_dt, dw,
                              status, ws, nws)


@pytest.mark.parametrize("kw,st", [
    (dict(dt=2), EINVAL), (dict(T=-1), EINVAL), (dict(d=20), EINVAL), (dict(d=0), EINVAL), (dict(V=0), EINVAL),
    (dict(V=1 << 23), EINVAL), (dict(d=1 << 23, ldx=1 << 23, lddx=1 << 23), EINVAL), (dict(x=None), EINVAL),
    (dict(w=None), EINVAL), (dict(targets=None), EINVAL), (dict(loss=None), EINVAL), (dict(status=None), EINVAL),
    (dict(dx=None), EINVAL), (dict(dw=None), EINVAL), (dict(ldx=16), EINVAL), (dict(ldx=28), EINVAL), (dict(lddx=23), EINVAL),
    (dict(scale=math.nan), EINVAL), (dict(scale=math.inf), EINVAL), (dict(dw_dt=2), EINVAL), (dict(dt=0, dw_dt=1), EINVAL),
    (dict(x=ctypes.c_void_p(4100)), EINVAL), (dict(w=ctypes.c_void_p(4104)), EINVAL), (dict(dx=ctypes.c_void_p(4104)), EINVAL),
    (dict(lddx=32), EINVAL), (dict(ldx=32), EINVAL),   # dx over rows of x that lie otherwise
    (dict(ws=None), EWORKSPACE), (dict(nws=64), EWORKSPACE), (dict(ws=ctypes.c_void_p(4104)), EWORKSPACE)], ids=str)
def test_loss_refuses(kw, st):
    assert _loss(B.lib(), **kw) == st


def test_loss_workspace_is_bounded():
    """Whatever T: one piece's exponentials (2 GiB), its copy of x, maxima and sums, partial sums."""
    q = B.moe_vocab_loss_workspace_bytes
    for dt in (0, 1):
        assert q(dt, 0, 64, 1000, dt) == q(dt, 0, 64, 1000) == 256
        assert q(dt, 1 << 20, 64, 131072, dt) <= (1 << 31) * 1.3
        assert q(dt, 1 << 20, 64, 131072) <= (1 << 28) * 1.1
    assert q(1, 1 << 20, 64, 131072, 1) - q(1, 1 << 20, 64, 131072, 0) == 131072 * 64 * 4   # fp32 sums of a bf16 dW
    assert q(1, 8192, 64, 131072, 1) == q(1, 8192, 64, 131072, 0)                           # one piece needs none
    assert q(2, 8, 64, 100) == q(1, -1, 64, 100) == q(1, 8, 60, 100) == q(1, 8, 64, 0) == q(0, 8, 64, 100, 1) == 0
