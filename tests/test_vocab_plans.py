"""The kernel choice of the vocabulary loss's products (plan.hpp, compiled for the host): what
large, small and ragged ones take, and that the shapes of the GPU tests reach every kernel."""
import ctypes
import os
import subprocess
import tempfile

import pytest

from test_gpu_vocab import SIZES, TILES
from tiles_util import CSRC

SRC = '''#include "plan.hpp"
using namespace moe;
extern "C" void product(int f32, int which, int M, int N, int K, int64_t lda, int64_t ldb, int mode, int* out) {
  const DensePlan d = plan_dense({f32 != 0, false, which == 0, which > 0, which == 2, M, N, K, lda, ldb, which == 0,
                                  which == 1 ? 64 : 16}, 256, mode);
  const int v[] = {d.kernel, d.h, d.n_mt, d.nt, d.splits, d.klen, vocab_few(f32 != 0, M, N, K, d)};
  for (int i = 0; i < 7; ++i) out[i] = v[i];
}
'''
BIG, MID, DEEP = range(3)


@pytest.fixture(scope="module")
def lib():
    tmp = tempfile.mkdtemp()
    src, so = os.path.join(tmp, "p.cpp"), os.path.join(tmp, "p.so")
    with open(src, "w") as f:
        f.write(SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", so], check=True)
    L = ctypes.CDLL(so)
    L.product.argtypes = [ctypes.c_int] * 5 + [ctypes.c_int64] * 2 + [ctypes.c_int, ctypes.c_void_p]
    return L


def plans(lib, T, d, V, f32, mode=0):
    """(kernel, height, tiles along M and N, ranges, their length, few) of the logits, dX and dW."""
    s = 4 if f32 else 2
    pitch = -(-V * s // 128) * 128
    out = []
    for which, (M, N, K, lda, ldb) in enumerate(((T, V, d, d * s, d * s), (T, d, V, pitch, d * s), (V, d, T, pitch, d * s))):
        o = (ctypes.c_int * 7)()
        lib.product(int(f32), which, M, N, K, lda, ldb, mode, o)
        out.append(tuple(o))
    return out


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("mode", [0, 1, 2])
def test_tiles_cover_the_products(lib, f32, mode):
    for T, d, V in [s[:3] for s in SIZES] + [(8192, 4096, 131072), (1, 4096, 131072), (65536, 64, 31)]:
        for which, (M, N, K) in enumerate(((T, V, d), (T, d, V), (V, d, T))):
            k, h, n_mt, nt, splits, klen, _ = plans(lib, T, d, V, f32, mode)[which]
            rows, cols = (256, 256) if k == BIG else (32 * h, 128)
            assert n_mt * rows >= M > 0 and nt * cols >= N and (nt - 1) * cols < N
            assert splits * klen >= K and (splits - 1) * klen < K and klen % (32 if f32 else 64) == 0
            assert not (f32 and k == BIG) and (mode == 0 or k != DEEP) and (which or splits == 1)
            if mode == 1 and not f32:
                assert k == BIG
            if mode == 2:
                assert k == MID


def test_the_gpu_tests_reach_every_kernel(lib):
    for f32 in (False, True):
        seen = [plans(lib, *s[:3], f32) for s in SIZES + TILES["f32" if f32 else "bf16"]]
        assert any(p[0][6] for p in seen) and not all(p[0][6] for p in seen)
        logits, dx, dw = ({p[i][:2] for p in seen if i or not p[0][6]} for i in range(3))
        if f32:
            assert logits >= {(MID, h) for h in range(1, 7)} | {(DEEP, 1), (DEEP, 2)}
            assert dx >= {(MID, 3), (DEEP, 1), (DEEP, 2), (DEEP, 4)} and dw >= {(MID, 4), (DEEP, 1), (DEEP, 2)}
        else:
            assert logits >= {(MID, h) for h in (1, 3, 4, 5, 6)} | {(DEEP, 1), (DEEP, 2), (BIG, 0)}
            assert dx >= {(DEEP, 2), (DEEP, 4)} and dw >= {(MID, 4), (BIG, 0)}
        assert any(p[1][4] > 16 for p in seen) and any(p[1][4] == 1 for p in seen)     # ranges of dX
        assert any(p[2][4] > 1 for p in seen)                                           # and of dW


def test_choices(lib):
    """Large products take 256x256 tiles; one token streams the weights; nine tokens of a large vocabulary
    do not; few rows on a long sum do."""
    assert [p[0] for p in plans(lib, 8192, 4096, 131072, False)] == [BIG] * 3
    assert plans(lib, 1, 4096, 131072, False)[0][6] and not plans(lib, 9, 4096, 131072, False)[0][6]
    assert plans(lib, 16, 2608, 1717, False)[0][6] and plans(lib, 32, 2608, 1717, True)[0][6]
    assert not plans(lib, 17, 2608, 1717, False)[0][6] and not plans(lib, 2, 1024, 50001, False)[0][6]
    assert plans(lib, 509, 2048, 50001, False)[0][:2] == (MID, 6)
