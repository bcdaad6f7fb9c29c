"""The 8-bit integer path on the GPU against the oracle: row quantisation
(every integer and scale equal), the grouped product (exact sums, so only the
roundings of the scaling are allowed), and the expert FFN made of both."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import dev, to_np
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# one rounding of the result to its type, relative
ROUND = {"bf16": 2.0 ** -8, "f32": U32}


def _d(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(dev())
    return t if dtype is None else t.to(dtype)


def _special_rows(x, rng):
    """Overwrites the first rows with what a quantiser gets wrong first."""
    R, n = x.shape
    rows = [np.zeros(n), np.full(n, 1e-41), rng.standard_normal(n) * 2.0 ** -140,
            rng.standard_normal(n) * 1e-30, rng.standard_normal(n) * 1e36,
            # quotients of exactly k + 1/2: scale 1 (largest 127), halves elsewhere
            np.concatenate([[127.0], rng.integers(-126, 126, n - 1) + 0.5]),
            np.concatenate([[254.0], 2 * rng.integers(-60, 60, n - 1) + 1.0]),
            np.where(np.arange(n) == n // 2, np.nan, 1.0), np.where(np.arange(n) == n - 1, np.inf, 2.0),
            np.where(np.arange(n) == 0, -np.inf, -3.0)]
    for i, r in enumerate(rows[:R]):
        x[i] = r
    return x


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n,pad", [(1, 8, 0), (3, 24, 8), (40, 1000, 0), (130, 2048, 24), (11, 2056, 0),
                                        (300, 4096, 0), (12, 8200, 40), (5, 14336, 0), (2, 40000, 8)])
def test_quantize_rows(dt, rows, n, pad):
    rng = np.random.default_rng(rows * n + pad)
    x = _special_rows(rng.standard_normal((rows, n)) * rng.uniform(0.1, 10, (rows, 1)), rng)
    wide = torch.full((rows + 1, n + pad), 7.0, dtype=DT[dt], device=dev())
    wide[:rows, :n] = _d(x.astype(np.float32)).to(DT[dt])
    w = B.quantized_width(n)
    q = torch.full((rows + 2, w), 99, dtype=torch.int8, device=dev())
    scale = torch.full((rows + 2,), 5.0, device=dev())
    B.moe_quantize_rows(wide[:rows, :n], q, scale)
    torch.cuda.synchronize()
    rq, rs = O.quantize_rows(to_np(wide[:rows, :n]))
    got = q.cpu().numpy()
    np.testing.assert_array_equal(got[:rows, :n], rq)
    assert not got[:rows, n:].any()
    np.testing.assert_array_equal(scale.cpu().numpy()[:rows], rs)
    assert (got[rows:] == 99).all() and (scale[rows:] == 5).all()      # nothing behind the last row


def test_quantize_many_values_next_to_borders():
    """Values one float32 step around every half of a scale that is no power of two."""
    amax = np.float32(0.7310586)
    s = amax * (np.float32(1) / np.float32(127))
    half = ((np.arange(-126, 126) + 0.5) * np.float64(s)).astype(np.float32)
    x = np.concatenate([[amax]] + [np.nextafter(half, np.float32(d), dtype=np.float32)
                                   for d in (-np.inf, np.inf)] + [half]).astype(np.float32)
    x = np.concatenate([x, np.zeros(-len(x) % 8, np.float32)])[None]
    q = torch.empty(1, B.quantized_width(x.shape[1]), dtype=torch.int8, device=dev())
    scale = torch.empty(1, device=dev())
    B.moe_quantize_rows(_d(x), q, scale)
    rq, rs = O.quantize_rows(x)
    np.testing.assert_array_equal(q.cpu().numpy()[:, :x.shape[1]], rq)
    assert scale.item() == rs[0]


def _quantised(rng, n, *lead):
    q = np.zeros((*lead, B.quantized_width(n)), np.int8)
    q[..., :n] = rng.integers(-127, 128, (*lead, n))
    return q, (rng.uniform(0.5, 2, lead) / 500).astype(np.float32)


def _layout(rows, slack):
    rows = np.asarray(rows, np.int64)
    off = O.exclusive_offsets(rows + np.asarray(slack, np.int64))
    return rows, off, int(off[-1]) + 3


SHAPES = [  # rows per expert, slack rows, K, N
    ([1], [0], 16, 8),
    ([0], [3], 32, 16),
    ([5, 0, 17], [0, 2, 1], 72, 40),
    ([300, 33, 1, 130], [1, 0, 7, 0], 136, 264),
    ([513], [0], 1032, 520),
    ([64, 64, 0, 250], [0, 0, 0, 6], 512, 1000),
    ([2] * 64, [0] * 64, 256, 72),
    ([300], [0], 256, 4104),
    ([300, 290], [0, 7], 1040, 4104),
]


@pytest.fixture(params=[0, 1, 2], ids=["auto", "tiles256", "tiles128"])
def tiles(request):
    B.moe_set_gemm_tiles(request.param)
    yield request.param
    B.moe_set_gemm_tiles(0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,slack,K,N", SHAPES)
@pytest.mark.parametrize("by_token", [False, True])
def test_matmul(tiles, rows, slack, K, N, dt, by_token):
    rng = np.random.default_rng(K + N)
    rows, off, R = _layout(rows, slack)
    E = len(rows)
    xq, xs = _quantised(rng, K, R)
    wq, ws = _quantised(rng, K, E, N)
    y = torch.full((R, N), 3.0, dtype=DT[dt], device=dev())
    ws_buf = B.workspace(B.moe_expert_matmul_i8_workspace_bytes(E, N, R), dev())
    src, k, scale = None, 1, xs
    if by_token:   # rows name picks t * k + j; the scales belong to the tokens
        k, T = 2, (R + 1) // 2
        src = rng.permutation(2 * T)[:R].astype(np.int32)
        scale = xs[:T].copy()
        xs = scale[src // k]
    B.moe_expert_matmul_i8(_d(off.astype(np.int32)), _d(rows.astype(np.int32)), _d(xq), _d(scale),
                           _d(wq), _d(ws), y, ws_buf, src=None if src is None else _d(src), k=k)
    got = to_np(y)
    used = np.zeros(R, bool)
    for e in range(E):
        r = slice(int(off[e]), int(off[e] + rows[e]))
        used[r] = True
        ref = O.matmul_i8(xq[r], xs[r], wq[e], ws[e])
        # the sum to float32, two products, the result's own type
        np.testing.assert_array_less(np.abs(got[r] - ref), np.abs(ref) * (3.01 * U32 + ROUND[dt]) + 1e-300)
    assert (got[~used] == 3).all()


def test_matmul_sums_are_exact():
    """The largest sum a call allows: K = 131072 products of 127 * 127."""
    K, N, R = 131072, 8, 3
    xq = torch.full((R, K), 127, dtype=torch.int8, device=dev())
    wq = torch.full((1, N, K), 127, dtype=torch.int8, device=dev())
    wq[0, 1] = -127
    y = torch.empty(R, N, device=dev())
    one = torch.ones(8, device=dev())
    B.moe_expert_matmul_i8(_d(np.array([0, R], np.int32)), _d(np.array([R], np.int32)), xq, one, wq,
                           one, y, B.workspace(B.moe_expert_matmul_i8_workspace_bytes(1, N, R), dev()))
    want = np.float32(K * 127 * 127)
    assert (y[:, 0] == want).all() and (y[:, 1] == -want).all()


def test_matmul_rows_that_are_not_numbers():
    """A row whose scale is NaN gives NaN and leaves its neighbours alone."""
    rng = np.random.default_rng(0)
    xq, xs = _quantised(rng, 64, 40)
    wq, ws = _quantised(rng, 64, 1, 24)
    xs[7] = np.nan
    y = torch.empty(40, 24, device=dev())
    B.moe_expert_matmul_i8(_d(np.array([0, 40], np.int32)), _d(np.array([40], np.int32)), _d(xq),
                           _d(xs), _d(wq), _d(ws), y,
                           B.workspace(B.moe_expert_matmul_i8_workspace_bytes(1, 24, 40), dev()))
    bad = torch.isnan(y)
    assert bad[7].all() and bad.sum() == 24


FFN = [  # rows per expert, slack, d, f
    ([1], [0], 8, 8),
    ([3, 0, 2], [0, 1, 0], 72, 40),
    ([40, 300, 0, 17], [2, 0, 3, 0], 136, 200),
    ([260], [0], 512, 1032),
]


@pytest.mark.parametrize("act", ["swiglu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,slack,d,f", FFN)
def test_ffn(tiles, rows, slack, d, f, dt, act):
    rng = np.random.default_rng(d + f)
    rows, off, R = _layout(rows, slack)
    E = len(rows)
    x = _d(rng.standard_normal((R, d)).astype(np.float32)).to(DT[dt])
    kd, kf = B.quantized_width(d), B.quantized_width(f)
    xq, xs = torch.empty(R, kd, dtype=torch.int8, device=dev()), torch.empty(R, device=dev())
    B.moe_quantize_rows(x, xq, xs)
    w1, s1 = _quantised(rng, d, E, f)
    w3, s3 = _quantised(rng, d, E, f) if act == "swiglu" else (None, None)
    w2, s2 = _quantised(rng, f, E, d)
    y = torch.full((R, d), 3.0, dtype=DT[dt], device=dev())
    code = B.MOE_BF16 if dt == "bf16" else B.MOE_F32
    ws = B.workspace(B.moe_ffn_fwd_i8_workspace_bytes(code, B.ACTS[act], E, d, f, R), dev())
    opt = lambda a: None if a is None else _d(a)
    B.moe_expert_ffn_fwd_i8(B.ACTS[act], _d(off.astype(np.int32)), _d(rows.astype(np.int32)), xq, xs,
                            _d(w1), _d(s1), opt(w3), opt(s3), _d(w2), _d(s2), y, ws)
    got, used = to_np(y), np.zeros(R, bool)
    xq, xs = xq.cpu().numpy()[:, :d], xs.cpu().numpy()
    for e in range(E):
        r = slice(int(off[e]), int(off[e] + rows[e]))
        used[r] = True
        if rows[e] == 0:
            continue
        part = lambda a, n: None if a is None else a[e][..., :n] if n else a[e]
        ref, slack_e = O.ffn_i8_bounds(xq[r], xs[r], part(w1, d), s1[e], part(w3, d),
                                       None if s3 is None else s3[e], part(w2, f), s2[e], act, dt)
        assert (np.abs(got[r] - ref) <= slack_e * 1.001 + np.abs(ref) * (4 * U32 + ROUND[dt]) + 1e-30).all()
    assert (got[~used] == 3).all()


@pytest.mark.parametrize("act", ["swiglu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("R", [2, 40, 300])
def test_ffn_shows_a_token_that_is_not_a_number(tiles, act, R):
    """A NaN or an infinity in one token: its whole output is NaN, the others' are numbers."""
    rng = np.random.default_rng(R)
    d, f = 64, 136
    x = rng.standard_normal((R, d)).astype(np.float32)
    x[1, 5] = np.nan if R != 40 else np.inf
    q, sc = torch.empty(R, 64, dtype=torch.int8, device=dev()), torch.empty(R, device=dev())
    B.moe_quantize_rows(_d(x), q, sc)
    (w1, s1), (w3, s3), (w2, s2) = _quantised(rng, d, 1, f), _quantised(rng, d, 1, f), _quantised(rng, f, 1, d)
    y = torch.empty(R, d, device=dev())
    g = act == "swiglu"
    B.moe_expert_ffn_fwd_i8(B.ACTS[act], _d(np.array([0, R], np.int32)), _d(np.array([R], np.int32)), q, sc, _d(w1),
                            _d(s1), _d(w3) if g else None, _d(s3) if g else None, _d(w2), _d(s2), y,
                            B.workspace(B.moe_ffn_fwd_i8_workspace_bytes(B.MOE_F32, B.ACTS[act], 1, d, f, R), dev()))
    bad = torch.isnan(y)
    assert bad[1].all() and bad.sum() == d


def test_empty_calls():
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=dev())
    q8 = lambda *s: torch.zeros(*s, dtype=torch.int8, device=dev())
    f = lambda *s: torch.ones(*s, device=dev())
    ws = B.workspace(1 << 20, dev())
    B.moe_quantize_rows(f(0, 16), q8(0, 16), f(0))
    B.moe_expert_matmul_i8(i32(0, 0), i32(0), q8(0, 16), f(0), q8(1, 8, 16), f(1, 8), f(0, 8), ws)
    B.moe_expert_ffn_fwd_i8(B.MOE_RELU, i32(0, 0), i32(0), q8(0, 16), f(0), q8(1, 8, 16), f(1, 8), None,
                            None, q8(1, 16, 16), f(1, 16), f(0, 16), ws)
    torch.cuda.synchronize()


@pytest.mark.parametrize("act", ["swiglu", "relu"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,rows,d,f", [(1, 2, [1, 0, 1], 136, 200),        # decoding: quantised in the second product
                                          (8, 2, [9, 7, 0], 64, 1000),
                                          (3, 1, [0, 0, 3], 72, 4104),
                                          (1, 2, [20, 1, 16], 72, 264),       # padded regions: more rows than picks
                                          (2, 1, [1, 1, 0], 16, 24576)])      # too wide for LDS
def test_ffn_few_rows(T, k, rows, d, f, dt, act):
    """Decoding, with scales by token: rows[e] need not be the picks alone."""
    rng = np.random.default_rng(T * d + f)
    rows, off, R = _layout(rows, [2, 0, 1])
    x = _d(rng.standard_normal((T, d)).astype(np.float32)).to(DT[dt])
    xq, xs = torch.empty(T, B.quantized_width(d), dtype=torch.int8, device=dev()), torch.empty(T, device=dev())
    B.moe_quantize_rows(x, xq, xs)
    src = rng.integers(0, T * k, R).astype(np.int32)
    w1, s1 = _quantised(rng, d, 3, f)
    w3, s3 = _quantised(rng, d, 3, f) if act == "swiglu" else (None, None)
    w2, s2 = _quantised(rng, f, 3, d)
    y = torch.full((R, d), 3.0, dtype=DT[dt], device=dev())
    code = B.MOE_BF16 if dt == "bf16" else B.MOE_F32
    ws = B.workspace(B.moe_ffn_fwd_i8_workspace_bytes(code, B.ACTS[act], 3, d, f, R), dev())
    opt = lambda a: None if a is None else _d(a)
    xd = xq[_d(src // k).long()]
    B.moe_expert_ffn_fwd_i8(B.ACTS[act], _d(off.astype(np.int32)), _d(rows.astype(np.int32)), xd, xs, _d(w1),
                            _d(s1), opt(w3), opt(s3), _d(w2), _d(s2), y, ws, src=_d(src), k=k)
    got, used = to_np(y), np.zeros(R, bool)
    q, sc = xd.cpu().numpy()[:, :d], xs.cpu().numpy()[src // k]
    for e in range(3):
        r = slice(int(off[e]), int(off[e] + rows[e]))
        used[r] = True
        if rows[e] == 0:
            continue
        part = lambda a, n: None if a is None else a[e][..., :n]
        ref, slack_e = O.ffn_i8_bounds(q[r], sc[r], part(w1, d), s1[e], part(w3, d),
                                       None if s3 is None else s3[e], part(w2, f), s2[e], act, dt)
        assert (np.abs(got[r] - ref) <= slack_e * 1.001 + np.abs(ref) * (4 * U32 + ROUND[dt]) + 1e-30).all()
    assert (got[~used] == 3).all()


def test_quantize_rows_far_apart():
    """Rows 64 MB apart, past 2^31 elements: the bits of contiguous rows."""
    x = torch.randn(140, 72, device=dev()).to(torch.bfloat16)
    far = torch.empty(140 << 25, dtype=torch.bfloat16, device=dev()).view(140, -1)[:, 8:80]
    far.copy_(x)
    out = []
    for t in (x, far):
        q, s = torch.empty(140, 80, dtype=torch.int8, device=dev()), torch.empty(140, device=dev())
        B.moe_quantize_rows(t, q, s)
        out.append((q, s))
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("each", [2, 40])
def test_weights_past_32_bits(tiles, each):
    """Five experts of 1 GiB of weights: the bits of a call for each expert alone (the sums are exact)."""
    E, K, N, R = 5, 16384, 65536, 5 * each
    wq = torch.randint(-127, 128, (E, N, K), dtype=torch.int8, device=dev())
    xq, xs = torch.randint(-127, 128, (R, K), dtype=torch.int8, device=dev()), torch.rand(R, device=dev())
    ws, y = torch.rand(E, N, device=dev()), torch.empty(R, N, device=dev())
    idx = lambda *v: torch.tensor(v, dtype=torch.int32, device=dev())
    buf = B.workspace(B.moe_expert_matmul_i8_workspace_bytes(E, N, R), dev())
    B.moe_expert_matmul_i8(idx(*range(0, R + 1, each)), idx(*[each] * E), xq, xs, wq, ws, y, buf)
    one = torch.empty(each, N, device=dev())
    for e in range(E):
        r = slice(e * each, (e + 1) * each)
        B.moe_expert_matmul_i8(idx(0, each), idx(each), xq[r], xs[r], wq[e:e + 1], ws[e:e + 1], one, buf)
        assert torch.equal(y[r], one), e
    # and a few columns of the last expert against whole numbers
    c = [0, N // 2 + 1, N - 1]
    exact = xq[-1].cpu().long() @ wq[-1, c].cpu().long().T
    ref = exact.double() * xs[-1].item() * ws[-1, c].cpu().double()
    assert ((y[-1, c].cpu().double() - ref).abs() <= 3.01 * U32 * ref.abs()).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,f", [([3, 0, 5], 72, 200), ([70, 1, 300], 136, 1000), ([500, 900, 40], 264, 520)])
def test_workspace_is_all_that_is_written(tiles, rows, d, f, dt):
    """The bytes behind a workspace of the queried size stay as they were."""
    rng = np.random.default_rng(d)
    E, R = len(rows), sum(rows)
    off = np.concatenate([[0], np.cumsum(rows)])
    xq, xs = _quantised(rng, d, R)
    w1, s1 = _quantised(rng, d, E, f)
    w2, s2 = _quantised(rng, f, E, d)
    code = B.MOE_BF16 if dt == "bf16" else B.MOE_F32
    size = B.moe_ffn_fwd_i8_workspace_bytes(code, B.MOE_RELU, E, d, f, R)
    buf = torch.full((size + (1 << 20),), 77, dtype=torch.uint8, device=dev())
    i = [_d(np.asarray(a, np.int32)) for a in (off, rows)]
    B.moe_expert_ffn_fwd_i8(B.MOE_RELU, *i, _d(xq), _d(xs), _d(w1), _d(s1), None, None, _d(w2), _d(s2),
                            torch.empty(R, d, dtype=DT[dt], device=dev()), buf[:size])
    assert (buf[size:] == 77).all()
    size = B.moe_expert_matmul_i8_workspace_bytes(E, f, R)
    buf = torch.full((size + (1 << 20),), 77, dtype=torch.uint8, device=dev())
    B.moe_expert_matmul_i8(*i, _d(xq), _d(xs), _d(w1), _d(s1), torch.empty(R, f, dtype=DT[dt], device=dev()), buf[:size])
    assert (buf[size:] == 77).all()
