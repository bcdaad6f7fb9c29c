"""The kernel choice of the dense block and of the int8 products (plan.hpp,
compiled for the host): what large, small and ragged products take, and that
the shapes of the GPU tests reach every kernel."""
import ctypes
import os
import subprocess
import tempfile

import pytest

from tiles_util import CSRC

SRC = '''#include "plan.hpp"
using namespace moe;
extern "C" void dense(int f32, int gated, int active, int km, int dw, int M, int N, int K, int64_t lda, int64_t ldb,
                      int mode, int* out) {
  const DensePlan d = plan_dense({f32 != 0, gated != 0, active != 0, km != 0, dw != 0, M, N, K, lda, ldb}, 256, mode);
  const int v[] = {d.kernel, d.h, d.n_mt, d.nt, d.splits, d.klen};
  for (int i = 0; i < 6; ++i) out[i] = v[i];
}
extern "C" int i8(int E, int64_t rows, int K, int N, int gated, int mode) {
  return plan_i8(E, rows, K, N, gated != 0, 256, mode);
}
'''
BIG, MID, DEEP = range(3)
I8_FEW, I8_DEEP32, I8_DEEP64, I8_DEEP128, I8_MID, I8_BIG = range(6)


@pytest.fixture(scope="module")
def lib():
    tmp = tempfile.mkdtemp()
    src, so = os.path.join(tmp, "p.cpp"), os.path.join(tmp, "p.so")
    with open(src, "w") as f:
        f.write(SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", so], check=True)
    L = ctypes.CDLL(so)
    L.dense.argtypes = [ctypes.c_int] * 8 + [ctypes.c_int64] * 2 + [ctypes.c_int, ctypes.c_void_p]
    L.i8.argtypes = [ctypes.c_int, ctypes.c_int64] + [ctypes.c_int] * 4
    return L


def block(T, d, f, f32):
    """name -> (gated, active, K-major B, weight gradient, M, N, K, pitches) of the block's products."""
    s, F = 4 if f32 else 2, 2 * f
    return {"h": (1, 1, 0, 0, T, f, d, d * s, d * s), "y": (0, 0, 0, 0, T, d, f, f * s, f * s),
            "da": (0, 1, 1, 0, T, f, d, d * s, f * s), "dx": (0, 0, 1, 0, T, d, F, F * s, d * s),
            "dw2": (0, 0, 1, 1, d, f, T, d * s, f * s), "dw13": (0, 0, 1, 1, F, d, T, F * s, d * s)}


def plan(lib, p, f32, mode=0):
    out = (ctypes.c_int * 6)()
    lib.dense(int(f32), *p, mode, out)
    return tuple(out)


SIZES = [(T, d, f) for T in (1, 17, 33, 300, 1021, 8192) for d, f in ((8, 8), (72, 200), (512, 1384), (4096, 14336))]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("mode", [0, 1, 2])
def test_plans_cover_their_products(lib, f32, mode):
    """Tiles cover M and N, the K ranges cover K in whole steps, none is empty; an activation's K stays whole."""
    for size in SIZES:
        for name, p in block(*size, f32).items():
            gated, active, _, dw, M, N, K = p[:7]
            kernel, h, n_mt, nt, splits, klen = plan(lib, p, f32, mode)
            rows, cols = (256, 256) if kernel == BIG else (32 * h, 128)
            assert (n_mt - 1) * 32 < M <= n_mt * rows and (nt - 1) * cols < N * (1 + gated) <= nt * cols, (size, name)
            assert klen % (32 if f32 else 64) == 0 and (splits - 1) * klen < K <= splits * klen, (size, name)
            assert splits == 1 or not active
            assert kernel != BIG or not f32
            assert f32 or mode == 0 or kernel == (BIG if mode == 1 else MID)
            assert 1 <= h <= 6 or kernel == BIG
            assert kernel != DEEP or h in (1, 2, 4)
            if dw and not f32:
                assert kernel == BIG or h == 4      # K-major tiles of 128 rows
            if dw and f32:
                assert h in (1, 2, 4)


def test_large_products_keep_the_large_tiles(lib):
    for name, p in block(8192, 4096, 14336, False).items():
        assert plan(lib, p, False)[0] == BIG and plan(lib, p, False)[4] == 1, name


def test_few_tiles_split_k(lib):
    for T in (32, 100, 257):
        for name in ("y", "dx"):
            assert plan(lib, block(T, 4096, 14336, False)[name], False)[4] > 1, (T, name)
        assert plan(lib, block(T, 1024, 2816, True)["dx"], True)[4] > 1


def test_int8_by_the_rows(lib):
    E, d, f = 8, 4096, 14336
    of = lambda rows: [lib.i8(E, rows, d, f, 1, 0), lib.i8(E, rows, f, d, 0, 0)]
    assert of(2) == [I8_FEW, I8_FEW]
    assert set(of(64)) <= {I8_DEEP32, I8_DEEP64}
    assert all(k >= I8_MID for k in of(2048) + of(8192))
    assert of(8192) == [I8_BIG, I8_MID]
    assert lib.i8(E, 2, d, f, 1, 1) == I8_BIG and lib.i8(E, 2, d, f, 1, 2) == I8_MID
    # more rows never go to the kernel for few, nor back to lower tiles
    for K, N in ((d, f), (1000, 2504), (14336, 4096)):
        for E in (1, 8, 64):
            seen = [lib.i8(E, r, K, N, 0, 0) for r in (1, 4, 16, 17, 64, 256, 1024, 4096, 16384)]
            assert I8_FEW not in seen[3:]


def test_the_gpu_tests_reach_every_kernel(lib):
    import test_gpu_gated as G
    import test_gpu_i8 as Q
    for f32 in (False, True):
        seen = set()
        for size in G.SHAPES + G.LARGER:
            for name, p in block(*size, f32).items():
                kernel, h, _, _, splits, _ = plan(lib, p, f32)
                seen.add((name, kernel, h if kernel == DEEP else 0, splits > 1))
        products = ("h", "y", "da", "dx", "dw2", "dw13")
        want = {(n, MID, 0) for n in products if not f32 or n in ("h", "y", "da", "dx")}
        want |= {(n, DEEP, h) for n in ("h", "y", "dx") for h in (1, 2, 4) if not (f32 and h == 4)}
        want |= {(n, DEEP, 4) for n in ("da", "dw2", "dw13") if not f32}
        want |= {(n, DEEP, h) for n in ("dw2", "dw13") for h in (1, 2) if f32}
        assert {s[:3] for s in seen} >= want, (f32, want - {s[:3] for s in seen})
        for name in ("y", "dx", "dw2", "dw13"):
            assert (name, True) in {(s[0], s[3]) for s in seen} and (name, False) in {(s[0], s[3]) for s in seen}
    # (256x256 tiles by the tests' forced mode; the mid tiles of the weight gradients in fp32 likewise)
    took = {lib.i8(len(rows), sum(rows) + sum(slack) + 3, -(-K // 16) * 16, N, 0, 0) for rows, slack, K, N in Q.SHAPES}
    assert took >= {I8_FEW, I8_DEEP32, I8_DEEP64, I8_DEEP128}, took


def test_the_gpu_tests_reach_every_kernel_of_the_transposed_weights(lib):
    """dX from the transposed copy of [W1; W3]: both operands K-contiguous."""
    import test_gpu_gated_copy as C
    seen = set()
    for T, d, f in C.SHAPES + C.LONG:
        kernel, h, _, _, splits, _ = plan(lib, (0, 0, 0, 0, T, d, 2 * f, 4 * f, 4 * f), False)
        seen |= {(kernel, h if kernel == DEEP else 0), ("split", splits > 1)}
    assert seen == {(BIG, 0), (MID, 0), (DEEP, 1), (DEEP, 2), (DEEP, 4), ("split", True), ("split", False)}
