"""The scale of a quantised row on the GPU: the header's product, for every bf16 maximum, and
the integers next to its half."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import dev
from paper_2205_01848_amd import quantize_rows
from test_oracle_blocks import OTHER_MAXIMA

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [8, 520, 4096])
def test_the_scale_is_the_product(dt, n):
    m = torch.arange(128, 256, dtype=torch.float32)
    x = torch.zeros(256, n)
    x[:128, 0], x[:128, 1], x[:128, n - 1] = m, m / 2, -m / 2
    x[128:] = x[:128] * 2.0 ** -9          # a power of two changes nothing but the scale
    q, s = quantize_rows(x.to(dt).to(dev()))
    rq, rs = O.quantize_rows(x.numpy())
    assert (s.cpu().numpy() == rs).all() and (q.cpu().numpy()[:, :n] == rq).all()
    assert (q[:128] == q[128:]).all()
    assert tuple(m[s.cpu()[:128] != m / 127].tolist()) == OTHER_MAXIMA   # (m / 127 on the host is the quotient)
    # as a tensor's division by a constant on this device
    assert torch.equal(s, x.to(dev()).abs().amax(1) / 127)


def test_rows_of_tensor_operations():
    """A program of tensor operations finds the same integers and scales."""
    g = torch.Generator(device=dev()).manual_seed(0)
    x = torch.randn(300, 1000, generator=g, device=dev())
    q, s = quantize_rows(x)
    scale = x.abs().amax(1) / 127
    ints = (x.double() / scale.double()[:, None]).round().clamp(-127, 127)
    assert torch.equal(s, scale) and torch.equal(q[:, :1000].double(), ints)
    assert not np.asarray(q[:, 1000:].cpu()).any()
