"""The loss of targets that have nearly all of the probability: its error is a few 2^-24 of 1, whatever
the size of the logits.

The logits are exact (5 a at the target, 0 elsewhere, a small whole number), so loss = log(1 + R), R =
(V - 1) exp(-5 a).  R is off by 64 U of itself: the exponent 5 a log2(e) <= 44 and its rounded constant and
sums, 44 ln 2 U each at most, and the sums of R.  The sum 1 + R is formed in at most 32 joins of
partial sums, each off by U; the logarithm and the sum with the maximum's difference (0) by 2 U of the loss."""
import numpy as np
import pytest
import torch

from gpu_util import dev, to_np
from paper_2205_01848_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(1, 1003), (6, 131072), (60, 5003), (300, 50001)])
@pytest.mark.parametrize("far", [0, 4096])
def test_error_of_a_small_loss(dt, T, V, far):
    """far: added to every logit of a row."""
    d, at = 64, V * 2 // 3
    a = np.arange(T) % 6 + 1
    x = torch.zeros(T, d, dtype=dt, device=dev())
    w = torch.zeros(V, d, dtype=dt, device=dev())
    x[:, 0] = torch.from_numpy(a).to(dev())
    w[at, 0] = 5
    x[:, 1], w[:, 1] = 64, far // 64
    target = torch.full((T,), at, dtype=torch.int32, device=dev())
    loss, lse, status = torch.empty(T, device=dev()), torch.empty(T, device=dev()), torch.zeros(1, dtype=torch.int32, device=dev())
    code = B.MOE_BF16 if dt == torch.bfloat16 else B.MOE_F32
    ws = B.workspace(B.moe_vocab_loss_workspace_bytes(code, T, d, V), dev())
    B.moe_vocab_loss(x, w, target, loss, lse, status, ws)
    want = np.log1p((V - 1) * np.exp(-5.0 * a))
    err = np.abs(to_np(loss) - want)
    assert (err <= 34 * U + 66 * U * want).all(), (err / U).max()
    top = 5.0 * a + far
    assert (np.abs(to_np(lse) - top - want) <= U * (top + want) + 34 * U + 66 * U * want).all()
