"""The dense gated block's dX from the transposed copy of [W1; W3], which the automatic mode
makes from 8192 tokens: against the oracle (test_gpu_gated's stages and bounds), over its
inputs, in a workspace of just the queried size."""
import pytest
import torch

import test_gpu_gated as G
from gpu_util import dev
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

# every kernel of that product, whole and with K split; 2f and d no multiples of 64 among them
SHAPES = [(1, 8, 8), (7, 72, 200), (33, 136, 264), (100, 40, 8200), (300, 520, 1384), (777, 136, 2056),
          (1030, 1032, 2056), (4100, 1032, 1032), (4100, 2056, 520)]
LONG = [(8200, 72, 136), (8200, 136, 520), (8200, 1032, 264)]


@pytest.fixture
def copy():
    B.moe_set_dx_weight_copy(2)
    yield
    B.moe_set_dx_weight_copy(0)


@pytest.fixture
def no_copy():
    B.moe_set_dx_weight_copy(1)
    yield
    B.moe_set_dx_weight_copy(0)


def _size(T, d, f):
    return B.moe_gated_ffn_bwd_workspace_bytes(B.MOE_BF16, T, d, f)


@pytest.mark.parametrize("T,d,f", SHAPES)
@pytest.mark.parametrize("mode", [0, 1, 2])
def test_gradients(copy, mode, T, d, f):
    try:
        B.moe_set_gemm_tiles(mode)
        G._check_block(T, d, f, "gelu_tanh", "bf16", 8)
    finally:
        B.moe_set_gemm_tiles(0)


@pytest.mark.parametrize("T,d,f", LONG)
def test_long_batches_make_the_copy(T, d, f):
    auto = _size(T, d, f)
    try:
        B.moe_set_dx_weight_copy(1)
        assert auto >= 4 * d * f and _size(T, d, f) < auto
    finally:
        B.moe_set_dx_weight_copy(0)
    G._check_block(T, d, f, "swiglu", "bf16", 8)


@pytest.mark.parametrize("T,d,f", LONG[:1])
def test_long_batches_without_it(no_copy, T, d, f):
    G._check_block(T, d, f, "swiglu", "bf16", 8)


@pytest.mark.parametrize("T,d,f", [(40, 64, 72), (777, 520, 264), (777, 40, 2056), (2056, 1032, 520)])
def test_outputs_over_inputs(copy, T, d, f):
    G.test_outputs_over_inputs(T, d, f, "bf16")


@pytest.mark.parametrize("T,d,f", [(1, 2056, 72), (40, 64, 72), (100, 40, 8200), (777, 136, 2056), (2056, 1032, 520)])
def test_workspace_is_all_that_is_written(copy, T, d, f):
    G.test_workspace_is_all_that_is_written(T, d, f, "bf16")


def test_a_workspace_without_the_copy_is_refused():
    """The query and the call are to see the same mode."""
    T, d, f = 40, 64, 72
    P = G._problem(T, d, f, "bf16")
    h = torch.zeros(3, T, f, dtype=torch.bfloat16, device=dev())
    dw = [torch.empty_like(P[n]) for n in ("w1", "w3", "w2")]
    ws = B.workspace(_size(T, d, f), dev())
    try:
        B.moe_set_dx_weight_copy(2)
        with pytest.raises(B.MoEError, match="workspace"):
            B.moe_gated_ffn_bwd(B.MOE_SWIGLU, P["x"], h, P["w1"], P["w3"], P["w2"], P["dy"],
                                torch.empty_like(P["dy"]), *dw, ws)
    finally:
        B.moe_set_dx_weight_copy(0)
