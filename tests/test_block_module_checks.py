"""What the modules around the linears refuse before they touch a device."""
import pytest
import torch


def test_shapes_and_types():
    from paper_2510_27527_b200.block import NVFP4LayerNorm, swiglu

    ln = NVFP4LayerNorm(64, device="cpu")
    for shape in ((3, 32), (64, 3), (), (2, 64, 1)):
        with pytest.raises(RuntimeError, match="64 features"):
            ln(torch.zeros(shape, dtype=torch.bfloat16))
    with pytest.raises(RuntimeError, match="float16"):
        ln(torch.zeros(3, 64, dtype=torch.float16))
    with pytest.raises(RuntimeError, match="CUDA device"):
        ln(torch.zeros(3, 64, dtype=torch.bfloat16))
    x = torch.zeros(3, 64, dtype=torch.bfloat16)
    for a, b in ((x, x[:2]), (x, x.float()), (x.half(), x.half())):
        with pytest.raises(RuntimeError, match="swiglu"):
            swiglu(a, b)
    with pytest.raises(RuntimeError, match="CUDA device"):
        swiglu(x, x)
