"""RMSNorm.quantized without a GPU: the rows of the last forward and no others."""
import pytest
import torch

from paper_2205_01848_amd import RMSNorm
from paper_2205_01848_amd import binding as B


@pytest.fixture
def norm(monkeypatch):
    monkeypatch.setattr(B, "moe_rms_norm_fwd", lambda *a, **kw: None)
    return RMSNorm(6, 24, torch.float32, quantized=True, device="cpu")


def test_the_last_forwards_rows(norm):
    w = torch.zeros(24)
    for rows in (6, 4, 0, 1, 6):
        norm.forward(torch.zeros(rows, 24), w)
        q, s = norm.quantized()
        assert q.shape == (rows, 32) and s.shape == (rows,) and q.data_ptr() == norm.q.data_ptr() * (rows > 0)
        for n in range(rows + 1):
            assert [t.shape[0] for t in norm.quantized(n)] == [n, n]
        for n in (-1, rows + 1):
            with pytest.raises(ValueError, match=f"the last forward left {rows}"):
                norm.quantized(n)


def test_before_a_forward(norm):
    with pytest.raises(ValueError, match="follow a forward"):
        norm.quantized()
    assert [t.shape[0] for t in norm.quantized(6)] == [6, 6]     # the buffers
    with pytest.raises(ValueError, match="left 6"):
        norm.quantized(7)
