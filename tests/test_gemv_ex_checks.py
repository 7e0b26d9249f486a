"""What nvfp4_gemv_ex and a status word are refused for, on the host."""
import ctypes

import pytest
import torch

from paper_2510_27527_b200 import binding as b


@pytest.mark.parametrize("opts,status", [((1, 0, 0), 4), ((-1, 0, 0), 4), ((0, 0, -1), 4), ((0, 1, 1000), 0), (None, 0)])
def test_options(opts, status):
    w = b.COperand(0x20000, 0x30000, 0x40000, 40, 64, 0, 1)
    o = None if opts is None else ctypes.byref(b.CGemmOpts(*opts))
    # (no tokens: nothing would be launched)
    assert b.lib.nvfp4_gemv_ex(0x10000, 64, 0, 64, ctypes.byref(w), None, None, 0, None, None, 0x50000, 0, 40, None, o, None, 0, None) == status


def test_arguments_are_counted():
    x = torch.zeros(1, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="14 arguments"):
        b._node.gemv(x, *[None] * 13)
