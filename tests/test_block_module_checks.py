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


def test_only_weights_on_a_device_are_frozen():
    from paper_2510_27527_b200.block import NVFP4MLP
    from paper_2510_27527_b200.module import NVFP4Linear

    with pytest.raises(RuntimeError, match="CUDA device"):
        NVFP4Linear(64, 32, device="cpu").frozen()
    with pytest.raises(RuntimeError, match="CUDA device"):
        NVFP4MLP(64, 128, device="cpu").frozen()


def test_an_mlps_outlier_channels_are_its_inputs():
    import numpy as np

    from paper_2510_27527_b200 import binding as b
    from paper_2510_27527_b200.block import NVFP4MLP

    cfg = b.LayerConfig(outliers=np.array([3, 60]), rht=True, seed=7)
    m = NVFP4MLP(64, 128, cfg, device="cpu")
    assert m.gate.cfg is cfg and m.up.cfg is cfg and m.down.cfg.n_out == 0 and m.down.cfg.rht and m.down.cfg.seed == 7
    other = b.LayerConfig(outliers=np.array([100]))
    assert NVFP4MLP(64, 128, cfg, other, device="cpu").down.cfg is other
