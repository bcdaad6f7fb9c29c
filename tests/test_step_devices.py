"""The calls around the layer run on their tensors' device and that device's current stream,
whichever device is current (as test_binding_devices has it of the layer's own calls)."""
import torch

from paper_2205_01848_amd import binding as B
from test_binding_devices import AllFar, seen  # noqa: F401


def _everything():
    z = torch.zeros
    x, w = z(4, 16), z(16)
    B.moe_rms_norm_fwd(x, w, 1e-5, y=z(4, 16))
    B.moe_rms_norm_bwd(x, w, z(4), x, z(4, 16), z(16), z(4096, dtype=torch.uint8))
    u8 = torch.uint8
    i32 = torch.int32
    B.moe_vocab_loss(x, z(9, 16), z(4, dtype=i32), z(4), z(4), z(1, dtype=i32), z(4096, dtype=u8), dx=z(4, 16), dw=z(9, 16))
    ts = B.AdamWList([B.AdamWTensor(z(16), z(16), z(16, dtype=u8), z(16, dtype=u8), m_exp=z(1, dtype=u8), v_exp=z(1, dtype=u8))])
    B.moe_adamw(ts, 0.1, 0.9, 0.99, 1e-8, 1)
    B.moe_adamw_unpack(ts, [[z(16), z(16)]])


def test_every_launch_is_on_the_tensors_device(seen):  # noqa: F811
    with AllFar():
        _everything()
    for name, stream, device in seen:
        assert (stream, device) == (1001, 1), name
    launches = {n for n, (_, args) in B.SIGNATURES.items() if args and args[0] is B._stream_p}
    assert launches == {n for n, _, _ in seen}
