"""A batch of fewer tokens than the layer was sized for, after a full one: the bits of a
layer of just those tokens, whatever the last batch left in the buffers."""
import pytest
import torch

from gpu_util import torch_dtype
from paper_2205_01848_amd import MoELayer
from test_gpu_layer_blocks import CAP, _gate, _setup

pytestmark = pytest.mark.gpu


def _of(L, wl, n, dt, sf=104, sact="swiglu"):
    """A layer of n tokens with the row budget of L."""
    return MoELayer(n, wl.d, wl.E, wl.k, wl.f, wl.act, torch_dtype(dt), L.rows_alloc, shared_f=sf, shared_act=sact)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 5, 131])
def test_shared_expert_on_fewer_tokens(dt, n):
    wl, dv, L = _setup(dt, "swiglu", backward=False)
    w = dv["w1"], dv["w3"], dv["w2"]
    L.forward(dv["x"], *w, **_gate(dv, wl), shared=dv["shared"])
    x = dv["dy"][:n].contiguous()
    y = L.forward(x, *w, **_gate(dv, wl), shared=dv["shared"])[:n]
    assert torch.equal(y, _of(L, wl, n, dt).forward(x, *w, **_gate(dv, wl), shared=dv["shared"]))
