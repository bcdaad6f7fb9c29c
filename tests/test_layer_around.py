"""RMSNorm, VocabLoss, AdamW and MoELayer.gradients without a GPU: what they refuse, what they pass
on (the library calls replaced by a record)."""
import pytest
import torch

from paper_2205_01848_amd import AdamW, MoELayer, RMSNorm, VocabLoss, rows_alloc_for
from paper_2205_01848_amd import binding as B

T, d, V = 6, 16, 9
f32, bf16 = torch.float32, torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    seen = []
    for name in ("moe_rms_norm_fwd", "moe_rms_norm_bwd", "moe_vocab_loss", "moe_adamw", "moe_adamw_unpack"):
        monkeypatch.setattr(B, name, lambda *a, _n=name, **kw: seen.append((_n, a, kw)))
    monkeypatch.setattr(B, "_device_of", lambda *a: 0)
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else t.data_ptr())
    return seen


def test_norm(calls):
    n = RMSNorm(T, d, f32, backward=True, device="cpu")
    x, a, w = torch.zeros(4, d), torch.zeros(4, d), torch.zeros(d)
    with pytest.raises(ValueError, match="follows a forward"):
        n.backward(x, w)
    assert n.forward(x, w, add=a).shape == (4, d)
    assert n.s.data_ptr() == n.sum.data_ptr() and n.s.shape == (4, d)
    assert n.backward(x, w).shape == (4, d)
    assert calls[1][1][0].data_ptr() == n.sum.data_ptr()
    n.forward(x, w)
    assert n.s is x and calls[2][2]["sum"] is None
    for bad in (torch.zeros(T + 1, d), torch.zeros(4, d + 8), torch.zeros(4, 1, d)):
        with pytest.raises(ValueError, match="the norm takes up to"):
            n.forward(bad, w)
    with pytest.raises(ValueError, match="without rows in 8 bits"):
        n.quantized()
    with pytest.raises(ValueError, match="without a backward"):
        RMSNorm(T, d, f32, device="cpu").backward(x, w)
    q, s = RMSNorm(T, 24, f32, quantized=True, device="cpu").quantized(4)
    assert q.shape == (4, 32) and s.shape == (4,)


def test_loss(calls):
    l = VocabLoss(T, d, V, bf16, backward=True, dw_dtype=bf16, device="cpu")
    assert l.dw.dtype == bf16 and VocabLoss(T, d, V, bf16, device="cpu").dx is None
    l.forward(torch.zeros(T, d), torch.zeros(V, d), torch.zeros(T))
    assert calls[0][2]["scale"] == 1 / T
    l.forward(torch.zeros(T, d), torch.zeros(V, d), torch.zeros(T), scale=0.0)
    assert calls[1][2]["scale"] == 0.0
    for x, w in ((torch.zeros(T - 1, d), torch.zeros(V, d)), (torch.zeros(T, d), torch.zeros(V + 1, d))):
        with pytest.raises(ValueError, match="x and w have shapes"):
            l.forward(x, w, torch.zeros(T))


def test_adamw(calls):
    big, small, vec = torch.zeros(100, 50, dtype=bf16), torch.zeros(8, 8, dtype=bf16), torch.zeros(5000)
    o = AdamW([(t, torch.zeros(t.shape)) for t in (big, small, vec)], bits=8, weight_decay=0.2)
    t = o.list.tensors
    assert [x.m.dtype for x in t] == [torch.uint8, f32, torch.uint8] and t[0].m_exp.numel() == 40
    assert [x.weight_decay for x in t] == [0.2, 0.2, 0.0]
    assert t[0].master is not None and t[2].master is None
    o.step(lr=0.5)
    o.step()
    assert [c[1][6] if len(c[1]) > 6 else c[2]["seed"] for c in calls] == [1, 2] and o.lr == 0.5
    assert calls[1][1][5] == 2
    assert [len(p) for p in o.moments()] == [2, 2, 2] and calls[2][0] == "moe_adamw_unpack"
    assert AdamW([(big, torch.zeros(100, 50))], master=False).list.tensors[0].master is None
    with pytest.raises(ValueError, match="8 or 32"):
        AdamW([], bits=16)
    with pytest.raises(B.MoEError, match="listed twice"):
        AdamW([(big, torch.zeros(100, 50)), (big, torch.zeros(100, 50))])
    memory = torch.zeros(64)
    AdamW([(torch.zeros(16), memory[:16]), (torch.zeros(16), memory[:16])])      # one gradient of two weights
    for p, g in ((memory[:16], memory[:16]), (memory[8:24], memory[:16]), (memory[:16], memory[8:24])):
        with pytest.raises(B.MoEError, match="overlap"):
            AdamW([(p, g)])
    with pytest.raises(B.MoEError, match="overlap"):        # another's weight inside a longer gradient
        AdamW([(torch.zeros(48), memory[:48]), (memory[20:28], torch.zeros(8))])
    with pytest.raises(B.MoEError, match="g holds"):
        AdamW([(big, torch.zeros(99, 50))])


def test_captured_schedule(calls):
    o = AdamW([(torch.zeros(8), torch.zeros(8))], lr=0.25, betas=(0.5, 0.75), captured=True)
    o.prepare()
    assert o.schedule[:3].tolist() == [0.25, 2.0, 2.0] and o.schedule.view(torch.int32)[3] == 1
    o.apply()
    assert calls[0][2]["schedule"] is o.schedule


def test_layer_gradients():
    E, k, f = 4, 2, 24
    L = MoELayer(T, d, E, k, f, "relu", f32, rows_alloc_for("exact", T, k, E), backward=True, device="cpu", shared_f=8)
    w1, w2, w_g = torch.zeros(E, f, d), torch.zeros(E, d, f), torch.zeros(E, d)
    sh = torch.zeros(8, d), torch.zeros(8, d), torch.zeros(d, 8)
    assert [g is h for (_, g), h in zip(L.gradients(w1, None, w2), (L.dw1, L.dw2))] == [True, True]
    every = L.gradients(w1, None, w2, w_g=w_g, shared=sh)
    assert [tuple(p.shape) for p, _ in every] == [tuple(g.shape) for _, g in every] and len(every) == 6
    with pytest.raises(ValueError, match="without a backward"):
        MoELayer(T, d, E, k, f, "relu", f32, 12, device="cpu").gradients(w1, None, w2)
    with pytest.raises(ValueError, match="without a gate"):
        MoELayer(T, d, E, k, f, "relu", f32, 12, backward=True, gate=False, device="cpu").gradients(w1, None, w2, w_g=w_g)
    with pytest.raises(ValueError, match="without a shared expert"):
        MoELayer(T, d, E, k, f, "relu", f32, 12, backward=True, device="cpu").gradients(w1, None, w2, shared=sh)
