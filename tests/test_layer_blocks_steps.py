"""The shared expert and the int8 forward inside MoELayer, on the host (no GPU: the library
calls are replaced by a record of their arguments): they work on the tokens of x, whatever
the layer's buffers hold behind them."""
import pytest
import torch

from paper_2205_01848_amd import MoELayer, rows_alloc_for
from paper_2205_01848_amd import binding as B

T, d, E, k, f = 8, 24, 4, 2, 32
CALLS = ["moe_gate_topk", "moe_quantize_rows", "moe_count", "moe_update_capacity", "moe_dispatch", "moe_route",
         "moe_expert_ffn_fwd", "moe_expert_ffn_fwd_i8", "moe_combine", "moe_gated_ffn_fwd"]


@pytest.fixture
def calls(monkeypatch):
    seen = []
    for name in CALLS:
        monkeypatch.setattr(B, name, lambda *a, _n=name, **kw: seen.append((_n, a, kw)))
    return seen


def _layer(cls=MoELayer, **kw):
    return cls(T, d, E, k, f, "relu", torch.float32, rows_alloc_for("dynamic", T, k, E, 5, 4), device="cpu", **kw)


def _args(calls, name):
    found = [(a, kw) for n, a, kw in calls if n == name]
    assert len(found) == 1, [n for n, _, _ in calls]
    return found[0]


SHARED = (torch.zeros(16, d), torch.zeros(16, d), torch.zeros(d, 16))


@pytest.mark.parametrize("n", [0, 1, 5])
@pytest.mark.parametrize("backward", [False, True])
def test_a_forward_of_fewer_tokens_has_its_shared_expert(calls, n, backward):
    L = _layer(shared_f=16, backward=backward)
    L.forward(torch.zeros(n, d), torch.zeros(E, f, d), None, torch.zeros(E, d, f), w_g=torch.zeros(E, d), shared=SHARED)
    a, kw = _args(calls, "moe_gated_ffn_fwd")
    assert a[1].shape == a[5].shape == kw["add"].shape == (n, d)
    assert a[5].data_ptr() == L.y.data_ptr() or n == 0
    assert a[6].numel() >= B.moe_gated_ffn_fwd_workspace_bytes(B.MOE_F32, n, d, 16)


def test_the_shared_workspace_of_fewer_tokens(calls):
    """Fewer tokens may split K into more ranges and so need more workspace than all of them."""
    most, wide, sf = 1500, 8192, 8192
    need = {n: B.moe_gated_ffn_fwd_workspace_bytes(B.MOE_BF16, n, wide, sf) for n in (1, 100, 1024, most)}
    assert need[1024] > need[most]
    L = MoELayer(most, wide, E, k, f, "relu", torch.bfloat16, 1, device="cpu", shared_f=sf)
    for n, least in need.items():
        L.shared_fwd(torch.zeros(n, wide, dtype=torch.bfloat16), (torch.zeros(sf, 1).expand(sf, wide), None, None))
        assert calls[-1][1][6].numel() >= least, n


class Experts:
    E, f, d = E, f, d
    w1 = s1 = w3 = s3 = w2 = s2 = None


@pytest.mark.parametrize("n", [0, 1, 5, T])
@pytest.mark.parametrize("kind", ["static", "dynamic", "policy"])
@pytest.mark.parametrize("cached", [False, True])
def test_int8_forward_of_fewer_tokens(calls, n, kind, cached):
    """None of the rows behind x's tokens is quantised, routed or combined."""
    L = _layer(shared_f=16)
    given = dict(ids=torch.zeros(n, k, dtype=torch.int32), weights=torch.zeros(n, k)) if cached else dict(w_g=torch.zeros(E, d))
    y = L.forward_i8(torch.zeros(n, d), Experts, capacity=(kind, 5, 4), **given, shared=SHARED)
    assert y.shape == (n, d) and (y.data_ptr() == L.y.data_ptr() or n == 0)
    x, q, scale = _args(calls, "moe_quantize_rows")[0]
    assert x.shape == (n, d) and q.shape == (n, 32) and scale.shape == (n,)
    a = _args(calls, "moe_dispatch" if kind == "policy" else "moe_route")[0]
    assert a[0].shape == (n, 16) and a[1].shape == (n, k)
    a, kw = _args(calls, "moe_expert_ffn_fwd_i8")
    assert a[4].shape == (n,) and kw["k"] == k
    a = _args(calls, "moe_combine")[0]
    assert a[1].shape == (n, k) and a[2].numel() >= n * k and a[3].shape == (n, d)
    a, kw = _args(calls, "moe_gated_ffn_fwd")
    assert a[1].shape == a[5].shape == kw["add"].shape == (n, d)


def test_int8_forward_refuses_other_shapes(calls):
    L, g = _layer(), dict(w_g=torch.zeros(E, d))
    for x in (torch.zeros(T + 1, d), torch.zeros(T, d - 8), torch.zeros(T, d + 8), torch.zeros(T * d)):
        with pytest.raises(ValueError, match="x has shape"):
            L.forward_i8(x, Experts, **g)
    for shape in ((T - 1, k), (T, k + 1), (T + 1, k), (T * k,)):
        with pytest.raises(ValueError, match="ids"):
            L.forward_i8(torch.zeros(T, d), Experts, ids=torch.zeros(*shape, dtype=torch.int32))
    assert not calls


@pytest.mark.parametrize("serve", [False, True])
def test_the_routing_workspace_of_fewer_tokens(calls, serve):
    """A short batch is routed by kernels of its own, which take more workspace than a longer one."""
    most, E, k = 3000, 64, 8
    need = {n: B.moe_route_workspace_bytes(n, E, k) for n in (1, 2048, most)}
    assert need[2048] > need[most]
    L = MoELayer(most, d, E, k, f, "relu", torch.float32, 64, device="cpu")
    experts = type("", (Experts,), dict(E=E))
    for n, least in need.items():
        x, calls[:] = torch.zeros(n, d), []
        if serve:
            L.forward_i8(x, experts, w_g=torch.zeros(E, d))
        else:
            L.route(x, L.ids, True, 1, 1)
        assert _args(calls, "moe_route")[0][16].numel() >= least, n


HOOKS = {"gate": "moe_gate_topk", "count": "moe_count", "capacity_dynamic": "moe_update_capacity",
         "combine": "moe_combine"}


@pytest.mark.parametrize("step", sorted(HOOKS))
@pytest.mark.parametrize("how", ["subclass", "instance"])
def test_overridden_steps_are_called(calls, step, how):
    own, hits = getattr(MoELayer, step), []

    def hook(self, *a, **kw):
        hits.append(step)
        return own(self, *a, **kw)

    L = _layer(type("Hooked", (MoELayer,), {step: hook}) if how == "subclass" else MoELayer)
    if how == "instance":
        setattr(L, step, hook.__get__(L))
    L.forward_i8(torch.zeros(T, d), Experts, w_g=torch.zeros(E, d))
    assert hits == [step]
    assert [n for n, _, _ in calls] == ["moe_gate_topk", "moe_quantize_rows", "moe_count", "moe_update_capacity",
                                        "moe_dispatch", "moe_expert_ffn_fwd_i8", "moe_combine"]
    # such a step knows the layer's T tokens only
    with pytest.raises(ValueError, match="x has shape"):
        L.forward_i8(torch.zeros(T - 1, d), Experts, w_g=torch.zeros(E, d))


@pytest.mark.parametrize("step", ["dispatch", "ffn_fwd"])
def test_steps_in_the_layer_type_are_refused(calls, step):
    """The int8 forward moves and multiplies int8 rows: it cannot call these."""
    L = _layer(type("Hooked", (MoELayer,), {step: lambda self, *a, **kw: None}))
    with pytest.raises(ValueError, match=step):
        L.forward_i8(torch.zeros(T, d), Experts, w_g=torch.zeros(E, d))
    assert not calls
