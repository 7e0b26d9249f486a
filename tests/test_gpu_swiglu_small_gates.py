"""SwiGLU where the sigmoid is a subnormal number and the products are not.

Tolerance: as in test_gpu_swiglu.py, and the sigmoid off by 2^-148 more (a subnormal result of a reciprocal good to a unit in the last place, 2^-149,
and its own rounding)."""
import numpy as np
import pytest
import torch

from oracle import block_ops as O
from paper_2510_27527_b200 import synth
from tests.block_util import BF16, device_rows, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("factor", [1.0, 2.0 ** 20, -(2.0 ** 100)])
@pytest.mark.parametrize("wide", [False, True])  # with gaps between the rows, and without
def test_between_the_smallest_normal_sigmoid_and_none(factor, wide):
    from paper_2510_27527_b200 import binding as b

    g = synth.round_to_bf16(-np.arange(86.0, 88.75, 0.25, dtype=np.float32).repeat(16).reshape(-1, 16))
    u, dh = (synth.round_to_bf16((np.random.default_rng(i).random(g.shape) + 0.5).astype(np.float32) * np.float32(f)) for i, f in ((1, factor), (2, 1.0)))
    put = (lambda v: device_rows(v, torch.bfloat16)) if wide else b.upload_bf16
    H, saved = b.nvfp4_swiglu_fwd(put(g), put(u))
    dG, dU = b.nvfp4_swiglu_bwd(put(dh), saved)
    g, u, dh = (v.astype(np.float64) for v in (g, u, dh))
    s, off = O._sigmoid(g), (16 + 1.2 * np.abs(g)) * 2.0 ** -23
    for got, want, unit in ((H, O.swiglu(g, u), np.abs(g * u)), (dG, O.swiglu_bwd(dh, g, u)[0], np.abs(dh * u) * (1 + np.abs(g))), (dU, O.swiglu_bwd(dh, g, u)[1], np.abs(dh * g))):
        tol = BF16 * np.abs(want) + (off * s + 2.0 ** -148) * unit * (1 + BF16) + 2.0 ** -134
        assert np.all(np.abs(host(got) - want) <= tol), float(np.abs(host(got) - want).max() / np.abs(want).max())


def test_below_it_nothing_is_left():
    from paper_2510_27527_b200 import binding as b

    g = torch.tensor([[-89.0, -100.0, -3e38]], device="cuda").bfloat16()
    H, saved = b.nvfp4_swiglu_fwd(g, torch.full_like(g, 3.0))
    dG, dU = b.nvfp4_swiglu_bwd(torch.ones_like(g), saved)
    assert not H.any() and not dG.any() and not dU.any()
