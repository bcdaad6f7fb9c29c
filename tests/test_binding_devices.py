"""Every entry point runs on its tensors' device and that device's current stream, whichever
device is current (no GPU: tensors that claim to live on device 1, a record in the library's
place)."""
import contextlib
import types

import pytest
import torch
from torch.overrides import TorchFunctionMode

from paper_2205_01848_amd import MoELayer, QuantizedExperts
from paper_2205_01848_amd import binding as B

T, d, E, k, f, R = 8, 16, 4, 2, 32, 24
bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32


class Far(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return 1


class AllFar(TorchFunctionMode):
    def __torch_function__(self, fn, kinds, args=(), kw=None):
        r = fn(*args, **(kw or {}))
        return r.as_subclass(Far) if type(r) is torch.Tensor else r


@pytest.fixture
def seen(monkeypatch):
    """(name, first argument or the policy calls' second, device current at the call) of every launch."""
    now, calls = [0], []

    @contextlib.contextmanager
    def device(i):
        was, now[0] = now[0], i
        yield
        now[0] = was

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *a: 4096

            def call(*a):
                s = a[1 if name.startswith("moe_policy") else 0]
                calls.append((name, getattr(s, "value", s), now[0]))
                return 0
            return call

    monkeypatch.setattr(B, "lib", Lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda i=None: types.SimpleNamespace(cuda_stream=1000 + (now[0] if i is None else i)))
    yield calls
    assert now == [0]


def _everything():
    z = torch.zeros
    x, w_g, dy = z(T, d), z(E, d), z(T, d)
    w = z(E, f, d), z(E, f, d), z(E, d, f)
    shared = z(f, d), z(f, d), z(d, f)
    L = MoELayer(T, d, E, k, f, "swiglu", f32, R, backward=True, device="cpu", shared_f=f)
    L.forward(x, *w, w_g=w_g, balance=0.1, shared=shared)                    # one call
    L.backward(x, dy, *w, w_g=w_g, shared=shared)
    L.forward(x, *w, w_g=w_g, rows="capacity")                               # the fallback, one call for the routing
    L.backward(x, dy, *w, target=z(T, d), rows="capacity")
    L.aggregate_spec()
    L.count = types.MethodType(MoELayer.count, L)                            # the steps one by one
    L.forward(x, *w, w_g=w_g)
    del L.count
    L.forward_i8(x, QuantizedExperts(*w), w_g=w_g, shared=shared)
    B.moe_expert_matmul_i8(L.offsets, L.fill, z(R, 16, dtype=torch.int8), z(R), z(E, f, 16, dtype=torch.int8),
                           z(E, f), z(R, f), z(4096, dtype=torch.uint8))
    B.moe_cached_weights(L.logits, L.ids, 0, z(T, k))
    B.moe_update_capacity(T, k, E, None, 5, 4, 0, capacity=L.capacity, offsets=L.offsets)   # tensors by name alone
    B.moe_cache_update(L.ids, L.ids, z(T, k, dtype=i32), z(1, dtype=i32))
    B.moe_dispatch_noalloc(x, L.ids, E, L.capacity, L.offsets, R, L.counts, L.fill, L.dest_row, L.src, L.x_disp,
                           L.status)
    p = B.CapacityPolicy(T, k, E, 1, (11, 10), (3, 2), [4] * E, device=1)
    p.begin(L.capacity, L.offsets)
    p.end(L.counts)


def test_every_launch_is_on_the_tensors_device(seen):
    with AllFar():
        _everything()
    for name, stream, device in seen:
        if name not in ("moe_policy_create", "moe_policy_destroy"):
            assert (stream, device) == (1001, 1), name
        elif name == "moe_policy_create":
            assert device == 1
    launches = {n for n, (_, args) in B.SIGNATURES.items()
                if args and args[0] is B._p and not n.startswith(("moe_policy", "moe_timing"))}
    launches |= {"moe_policy_begin", "moe_policy_end"}
    assert launches <= {n for n, _, _ in seen}, launches - {n for n, _, _ in seen}


def test_a_policy_of_another_device(seen):
    p = B.CapacityPolicy(T, k, E, 1, (11, 10), (3, 2), [4] * E)
    with AllFar(), pytest.raises(B.MoEError, match="device 1, the policy was made for 0"):
        p.end(torch.zeros(E, dtype=i32))
