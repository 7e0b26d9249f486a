"""What a change of type or device does to the buffers of a frozen module."""
import torch


def test_types_stay_and_devices_follow():
    from paper_2510_27527_b200 import block

    for cls in (block.NVFP4FrozenLinear, block.NVFP4FrozenMLP):
        m = cls.__new__(cls)
        torch.nn.Module.__init__(m)
        for n, t in (("a", torch.bfloat16), ("b", torch.float32), ("c", torch.uint8), ("d", torch.int32)):
            m.register_buffer(n, torch.ones(4, dtype=t))
        m.register_buffer("e", None)
        types = lambda: [m.a.dtype, m.b.dtype, m.c.dtype, m.d.dtype]  # noqa: E731
        want = types()
        for change in (m.half, m.double, m.float, m.bfloat16, lambda: m.to(torch.float16)):
            change()
            assert types() == want and bool((m.a == 1).all())
        m.to("meta", torch.float16)
        assert types() == want and {b.device.type for b in m.buffers()} == {"meta"}
