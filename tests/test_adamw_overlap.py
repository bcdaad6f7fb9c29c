"""AdamWList refuses arrays that overlap also where they are one tensor object."""
import pytest
import torch

from paper_2205_01848_amd import binding as B

f32, bf16, u8 = torch.float32, torch.bfloat16, torch.uint8


@pytest.fixture(autouse=True)
def host(monkeypatch):
    monkeypatch.setattr(B, "_device_of", lambda *a: 0)
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else t.data_ptr())


def arrays(bits, n=128):
    p = dict(p=torch.zeros(n, dtype=bf16), g=torch.zeros(n, dtype=bf16), master=torch.zeros(n))
    if bits == 32:
        return dict(p, m=torch.zeros(n), v=torch.zeros(n))
    return dict(p, **{k: torch.zeros(1 if "exp" in k else n, dtype=u8) for k in ("m", "v", "m_exp", "v_exp")})


@pytest.mark.parametrize("bits", [8, 32])
def test_one_object_in_two_places(bits):
    kw = arrays(bits)
    B.AdamWList([B.AdamWTensor(**kw)])
    pairs = [(a, b) for a in kw for b in kw if a < b and kw[a].dtype == kw[b].dtype and kw[a].numel() == kw[b].numel()]
    if bits == 32:
        kw["g"] = torch.zeros(128)           # of float32 gradients
        pairs = [p for p in pairs if "g" not in p] + [(a, "g") for a in ("m", "v", "master")]
    assert len(pairs) == (3 if bits == 8 else 6)
    for a, b in pairs:
        for src, to in ((a, b), (b, a)):
            with pytest.raises(B.MoEError, match="overlap"):
                B.AdamWList([B.AdamWTensor(**dict(kw, **{to: kw[src]}))])


def test_weight_that_is_its_gradient_or_anothers():
    n = 16
    p, m, v = (torch.zeros(n) for _ in range(3))
    t = lambda p, g: B.AdamWTensor(p, g, torch.zeros(n), torch.zeros(n))
    with pytest.raises(B.MoEError, match="overlap"):
        B.AdamWList([t(p, p)])
    with pytest.raises(B.MoEError, match="overlap"):
        B.AdamWList([t(p, m), t(m, v)])
    with pytest.raises(B.MoEError, match="overlap"):
        B.AdamWList([B.AdamWTensor(p, m, m, v)])
    B.AdamWList([t(p, v), t(m, v)])          # one gradient of two weights
