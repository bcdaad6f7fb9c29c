"""AdamW's weight decay where lr weight_decay is next to the steps of float32 below 1."""
import numpy as np
import pytest
import torch

from gpu_util import dev, to_np
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _decayed(p, lr, wd, bits, master):
    n = p.numel()
    z = lambda k: torch.zeros(k, dtype=torch.uint8 if bits == 8 else torch.float32, device=dev())
    exp = dict(m_exp=z(B.adamw_blocks(n)), v_exp=z(B.adamw_blocks(n))) if bits == 8 else {}
    t = B.AdamWTensor(p.bfloat16() if master else p.clone(), torch.zeros(n, device=dev()), z(n), z(n),
                      master=p.clone() if master else None, weight_decay=wd, **exp)
    B.moe_adamw(B.AdamWList([t]), lr, 0.9, 0.95, 1e-8, 10)
    return t.master if master else t.p


@pytest.mark.parametrize("lr,wd", [(1e-5, 0.01), (3e-5, 0.01), (1e-6, 0.1), (2e-7, 0.1), (3e-4, 0.1)])
@pytest.mark.parametrize("bits,master", [(32, False), (8, False), (32, True)])
def test_a_weight_decays_by_its_own_rate(lr, wd, bits, master):
    """Gradients and moments of 0: p (1 - lr wd), of which p is the nearest float32: half of its last
    place, and for lr and wd, rounded to float32, 4 U of the decay."""
    p = torch.randn(1 << 16, generator=torch.Generator().manual_seed(0)).to(dev())
    p0, got = to_np(p), to_np(_decayed(p, lr, wd, bits, master))
    want = p0 * (1 - lr * wd)
    half = np.spacing(np.abs(want).astype(np.float32)).astype(np.float64) / 2
    assert (np.abs(got - want) <= half + 4 * U * lr * wd * np.abs(p0)).all()


def test_infinite_weights_stay_what_they_are():
    """(a bias of -inf turns an expert off; 0 (-inf) would make it NaN)"""
    p = torch.tensor([np.inf, -np.inf, 0.0, -0.0], device=dev())
    for wd in (0.0, 0.1):
        got = _decayed(p, 1e-3, wd, 32, False)
        assert torch.equal(got, p)
