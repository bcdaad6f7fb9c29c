"""What the int8 products and the dense gated block refuse, on the CPU: the
binding before any device access, the C entry points before any launch."""
import ctypes

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


QUANT = dict(x=z(5, 24), q=z(5, 32, dt=i8), scale=z(5))
MATMUL = dict(offsets=z(3, dt=i32), rows=z(2, dt=i32), xq=z(9, 32, dt=i8), x_scale=z(9),
              wq=z(2, 16, 32, dt=i8), w_scale=z(2, 16), y=z(9, 16), ws=z(256, dt=u8))
FFN = dict(act=B.MOE_SWIGLU, offsets=z(3, dt=i32), rows=z(2, dt=i32), xq=z(9, 32, dt=i8), x_scale=z(9),
           w1q=z(2, 16, 32, dt=i8), w1_scale=z(2, 16), w3q=z(2, 16, 32, dt=i8), w3_scale=z(2, 16),
           w2q=z(2, 24, 16, dt=i8), w2_scale=z(2, 24), y_disp=z(9, 24), ws=z(256, dt=u8))
GATED = dict(act=B.MOE_RELU, x=z(5, 24), w1=z(16, 24), w3=z(16, 24), w2=z(24, 16), y=z(5, 24),
             ws=z(256, dt=u8))
GRAD = dict(act=B.MOE_RELU, x=z(5, 24), h_save=z(3, 5, 16), w1=z(16, 24), w3=z(16, 24), w2=z(24, 16),
            dy=z(5, 24), dx=z(5, 24), dw1=z(16, 24), dw3=z(16, 24), dw2=z(24, 16), ws=z(256, dt=u8))
CALLS = [(B.moe_quantize_rows, QUANT), (B.moe_expert_matmul_i8, MATMUL), (B.moe_expert_ffn_fwd_i8, FFN),
         (B.moe_gated_ffn_fwd, GATED), (B.moe_gated_ffn_bwd, GRAD)]


@pytest.mark.parametrize("fn,kw", CALLS, ids=lambda v: getattr(v, "__name__", ""))
def test_sizes_that_fit_reach_the_device_check(fn, kw):
    passes_checks(fn, **kw)


@pytest.mark.parametrize("fn,kw,name", [(fn, kw, n) for fn, kw in CALLS for n, t in kw.items()
                                        if torch.is_tensor(t) and n not in ("ws", "x", "xq", "wq", "w1q", "w1", "w2q")])
def test_every_operand_too_small(fn, kw, name):
    """One row (or element) less than the call reads or writes."""
    t = kw[name]
    with pytest.raises(B.MoEError, match=f"{name}"):
        fn(**dict(kw, **{name: t[:-1] if t.dim() < 3 else t[:, :-1].contiguous()}))


@pytest.mark.parametrize("fn,kw,name", [(fn, kw, n) for fn, kw in CALLS for n, t in kw.items()
                                        if torch.is_tensor(t) and n not in ("ws", "x", "y", "y_disp")])
def test_every_operand_of_another_type(fn, kw, name):
    with pytest.raises(B.MoEError):
        fn(**dict(kw, **{name: kw[name].double()}))


def test_layer_types():
    refuses("unsupported layer dtype", B.moe_quantize_rows, **dict(QUANT, x=z(5, 24, dt=torch.float16)))
    refuses("unsupported layer dtype", B.moe_expert_matmul_i8, **dict(MATMUL, y=z(9, 16, dt=torch.float16)))
    passes_checks(B.moe_expert_matmul_i8, **dict(MATMUL, y=z(9, 16, dt=bf16)))


def test_rows_of_wider_tensors():
    passes_checks(B.moe_quantize_rows, **dict(QUANT, x=z(5, 40)[:, :24]))
    refuses("contiguous", B.moe_quantize_rows, **dict(QUANT, x=z(24, 5).T))
    refuses("apart", B.moe_quantize_rows, **dict(QUANT, x=z(1, 24).expand(5, 24)))
    refuses("apart", B.moe_quantize_rows, **dict(QUANT, x=z(5, 27)[:, :24]))
    refuses("shape", B.moe_gated_ffn_fwd, **dict(GATED, y=z(5, 32)))
    passes_checks(B.moe_gated_ffn_fwd, **dict(GATED, y=z(5, 32)[:, :24], add=z(5, 48)[:, :24]))
    refuses("add", B.moe_gated_ffn_fwd, **dict(GATED, add=z(4, 24)))


def test_picks_instead_of_rows():
    """With src the scales belong to tokens; src itself names every row."""
    passes_checks(B.moe_expert_matmul_i8, **dict(MATMUL, src=z(9, dt=i32), k=2, x_scale=z(3)))
    refuses("src holds", B.moe_expert_matmul_i8, **dict(MATMUL, src=z(8, dt=i32), k=2))
    refuses("k picks", B.moe_expert_matmul_i8, **dict(MATMUL, src=z(9, dt=i32), k=0))
    refuses("x_scale", B.moe_expert_ffn_fwd_i8, **dict(FFN, src=z(9, dt=i32), k=2, x_scale=None))


def test_widths_and_optional_operands():
    refuses("rows of 32 bytes, expected 48", B.moe_expert_ffn_fwd_i8,
            **dict(FFN, w2q=z(2, 40, 16, dt=i8), w2_scale=z(2, 40), y_disp=z(9, 40)))
    refuses("w3q is required", B.moe_expert_ffn_fwd_i8, **dict(FFN, w3q=None))
    passes_checks(B.moe_expert_ffn_fwd_i8, **dict(FFN, act=B.MOE_RELU, w3q=None, w3_scale=None))
    passes_checks(B.moe_gated_ffn_fwd, **dict(GATED, h_save=z(3, 5, 16)))
    refuses("h_save holds", B.moe_gated_ffn_fwd, **dict(GATED, h_save=z(2, 5, 16)))
    refuses("dw3", B.moe_gated_ffn_bwd, **dict(GRAD, dw3=z(16, 24, dt=bf16)))


def _c(name, **change):
    """The C entry point on made-up addresses (never read: each call is refused)."""
    p = ctypes.c_void_p
    at = p(1 << 20)
    order = {
        "moe_quantize_rows": dict(stream=None, dt=1, rows=5, n=24, x=at, ldx=24, q=at, scale=at),
        "moe_expert_matmul_i8": dict(stream=None, dt=1, E=2, K=32, N=16, offsets=at, rows=at, R=9, xq=at,
                                     x_scale=at, src=None, T=0, k=1, wq=at, w_scale=at, y=at, ws=at,
                                     bytes=0),
        "moe_expert_ffn_fwd_i8": dict(stream=None, dt=1, act=2, E=2, d=24, f=16, offsets=at, rows=at, R=9,
                                      xq=at, x_scale=at, src=None, T=0, k=1, w1=at, s1=at, w3=at, s3=at,
                                      w2=at, s2=at, y=at, ws=at, bytes=0),
        "moe_gated_ffn_fwd": dict(stream=None, dt=1, act=2, T=5, d=24, f=16, x=at, ldx=24, w1=at, w3=at,
                                  w2=at, add=None, ldadd=0, h=None, y=at, ldy=24, ws=at, bytes=0),
        "moe_gated_ffn_bwd": dict(stream=None, dt=1, act=2, T=5, d=24, f=16, x=at, ldx=24, h=at, w1=at,
                                  w3=at, w2=at, dy=at, lddy=24, add=None, ldadd=0, dx=at, lddx=24, dw=0,
                                  dw1=at, dw3=at, dw2=at, ws=at, bytes=0),
    }[name]
    assert set(change) <= set(order), change
    return getattr(B.lib(), name)(*dict(order, **change).values())


ODD = ctypes.c_void_p((1 << 20) + 8)   # not on 16 bytes


@pytest.mark.parametrize("change", [dict(dt=2), dict(rows=-1), dict(n=0), dict(n=20), dict(n=131080),
                                    dict(ldx=16), dict(ldx=28), dict(x=None), dict(q=None),
                                    dict(scale=None), dict(x=ODD), dict(q=ODD)])
def test_c_quantize(change):
    assert _c("moe_quantize_rows", **change) == EINVAL


@pytest.mark.parametrize("change", [dict(dt=2), dict(E=0), dict(E=65), dict(K=0), dict(K=24), dict(K=131088),
                                    dict(N=0), dict(N=12), dict(R=-1), dict(R=1 << 31), dict(offsets=None),
                                    dict(rows=None), dict(xq=None), dict(x_scale=None), dict(wq=None),
                                    dict(w_scale=None), dict(y=None), dict(xq=ODD), dict(wq=ODD), dict(y=ODD),
                                    dict(src=ODD, T=-1), dict(src=ODD, T=4, k=0)])
def test_c_matmul(change):
    assert _c("moe_expert_matmul_i8", **change) == EINVAL


@pytest.mark.parametrize("change", [dict(dt=2), dict(act=3), dict(E=0), dict(E=65), dict(d=12), dict(f=12),
                                    dict(d=131080), dict(f=131080), dict(R=-1), dict(offsets=None),
                                    dict(rows=None), dict(xq=None), dict(x_scale=None), dict(w1=None),
                                    dict(s1=None), dict(w3=None), dict(s3=None), dict(w2=None), dict(s2=None),
                                    dict(y=None), dict(xq=ODD), dict(w1=ODD), dict(w3=ODD), dict(w2=ODD),
                                    dict(y=ODD), dict(src=ODD, T=-1), dict(src=ODD, T=4, k=0)])
def test_c_ffn(change):
    assert _c("moe_expert_ffn_fwd_i8", **change) == EINVAL


@pytest.mark.parametrize("change", [dict(dt=2), dict(act=3), dict(T=-1), dict(d=12), dict(f=12), dict(ldx=16),
                                    dict(ldx=28), dict(ldy=16), dict(ldx=1 << 23), dict(add=ODD, ldadd=24),
                                    dict(add=ctypes.c_void_p(1 << 20), ldadd=16), dict(x=None), dict(w1=None),
                                    dict(w3=None), dict(w2=None), dict(y=None), dict(x=ODD), dict(w1=ODD),
                                    dict(w3=ODD), dict(w2=ODD), dict(y=ODD), dict(h=ODD)])
def test_c_gated_fwd(change):
    assert _c("moe_gated_ffn_fwd", **change) == EINVAL


@pytest.mark.parametrize("change", [dict(dt=2), dict(act=3), dict(T=-1), dict(d=12), dict(f=12), dict(ldx=16),
                                    dict(lddy=16), dict(lddx=28), dict(dw=2), dict(dt=0, dw=1), dict(x=None),
                                    dict(h=None), dict(w1=None), dict(w3=None), dict(w2=None), dict(dy=None),
                                    dict(dx=None), dict(dw1=None), dict(dw3=None), dict(dw2=None), dict(h=ODD),
                                    dict(dy=ODD), dict(dx=ODD), dict(dw1=ODD), dict(dw3=ODD), dict(dw2=ODD),
                                    dict(add=ODD, ldadd=24), dict(add=ctypes.c_void_p(1 << 20), ldadd=16)])
def test_c_gated_bwd(change):
    assert _c("moe_gated_ffn_bwd", **change) == EINVAL


@pytest.mark.parametrize("name", ["moe_expert_matmul_i8", "moe_expert_ffn_fwd_i8", "moe_gated_ffn_fwd",
                                  "moe_gated_ffn_bwd"])
def test_c_workspaces(name):
    assert _c(name) == EWORKSPACE
    assert _c(name, ws=None, bytes=1 << 30) == EWORKSPACE
    assert _c(name, ws=ODD, bytes=1 << 30) == EWORKSPACE


def test_workspace_queries():
    q = B.lib()
    assert q.moe_expert_matmul_i8_workspace_bytes(2, 16, 9) > 0
    assert q.moe_expert_matmul_i8_workspace_bytes(0, 16, 9) == 0
    assert q.moe_expert_matmul_i8_workspace_bytes(2, 12, 9) == 0
    assert q.moe_ffn_fwd_i8_workspace_bytes(1, 2, 2, 24, 16, 9) > 0
    assert q.moe_ffn_fwd_i8_workspace_bytes(1, 3, 2, 24, 16, 9) == 0
    assert q.moe_gated_ffn_fwd_workspace_bytes(1, 5, 24, 16) > 0
    assert q.moe_gated_ffn_bwd_workspace_bytes(1, 5, 24, 12) == 0
    assert B.quantized_width(24) == q.moe_quantized_width(24) == 32
    assert all(B.quantized_width(n) == q.moe_quantized_width(n) for n in range(0, 300))
    assert q.moe_quantized_width(-1) == 0


@pytest.mark.parametrize("dt,rows", [(B.MOE_BF16, 16), (B.MOE_F32, 32)])
def test_a_forced_tile_mode_holds_for_few_tokens_too(dt, rows):
    """The automatic mode streams the weights of a few tokens' forward and needs room for A
    alone; a forced mode runs its tiles, which split K and need room for partial sums."""
    d, f = 4096, 14336
    size = lambda T: B.moe_gated_ffn_fwd_workspace_bytes(dt, T, d, f)
    a = lambda T: -(-T * f * (2 if dt == B.MOE_BF16 else 4) // 256) * 256
    try:
        for mode in (0, 1, 2):
            B.moe_set_gemm_tiles(mode)
            for T in (1, rows):
                assert (size(T) > a(T) + 256) == (mode != 0), (mode, T)
            assert size(rows + 1) > a(rows + 1) + 256, mode
    finally:
        B.moe_set_gemm_tiles(0)
