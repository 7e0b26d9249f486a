"""nvfp4_gemv on tokens far from 1: FP16 in between, and powers of two that are not subnormal numbers where the result is none.

Tolerance of an FP32 result: 2^-15 of sum_k |x_k w_k| as in test_gpu_gemv.py, and where numbers are subnormal half a step, 2^-150, of each of at most
64 sums. BF16's smallest step is 2^-133."""
import numpy as np
import pytest
import torch

from oracle import nvfp4_oracle as orc
from paper_2510_27527_b200 import synth
from tests.block_util import BF16, device_rows, host
from tests.gpu_util import upload_operand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gs", [0, 1, 2])
@pytest.mark.parametrize("M", [1, 2, 3, 6, 16, 32])
@pytest.mark.parametrize("exponent", [-126, -120, -116, -112, -108, -107, -104, -90, 60, 110, 111])
def test_tokens_of_any_magnitude(exponent, M, gs):
    from paper_2510_27527_b200 import binding as b

    N, K = 96, 640
    q = orc.quantize(synth.weights(N, K, 1), orc.AXIS_ROW, orc.RTN, gs, 0, 2)
    W, w = upload_operand(q, b), orc.dequantize(q)[:, :K]
    x = synth.round_to_bf16((synth.activations(M, K, 3, n_outlier=3, factor=30.0)[0] * 2.0 ** exponent).astype(np.float32))
    X = device_rows(x, torch.bfloat16)
    want, absdot = x.astype(np.float64) @ w.T, np.abs(x).astype(np.float64) @ np.abs(w).T
    for dt, last, step in ((b.DT_F32, 0.0, 0.0), (b.DT_BF16, BF16, 2.0 ** -134)):
        y = host(b.nvfp4_gemv(X, W, dt))
        tol = (2.0 ** -15 * absdot + 64 * 2.0 ** -150) * (1 + last) + last * np.abs(want) + step
        bad = np.abs(y - want) > tol
        assert not bad.any(), (int(bad.sum()), float((np.abs(y - want) / np.abs(want)).max()))


@pytest.mark.parametrize("M", [1, 2, 3, 6, 16])
def test_powers_of_two_of_a_token_are_exact(M):
    """Scaled tokens give scaled results, bit for bit, as long as nothing in it is subnormal."""
    from paper_2510_27527_b200 import binding as b

    W = b.nvfp4_quantize(torch.randn(100, 512, device="cuda").bfloat16())
    x = torch.randn(M, 512, device="cuda").clamp(-4, 4).bfloat16()
    x[x.abs() < 2.0 ** -8] = 0
    want = b.nvfp4_gemv(x, W, b.DT_F32).double()
    for e in (-110, -101, -64, -1, 1, 2, 3, 63, 110):
        assert torch.equal(b.nvfp4_gemv(x * 2.0 ** e, W, b.DT_F32).double(), want * 2.0 ** e)


def test_the_largest_numbers():
    """BF16's largest value in every place of an instruction, and weights that sum to little."""
    from paper_2510_27527_b200 import binding as b

    top = float(torch.finfo(torch.bfloat16).max)
    w = torch.full((40, 256), 2.0 ** -30, device="cuda").bfloat16()
    W = b.nvfp4_quantize(w)
    for M in (1, 3, 9, 20):
        x = torch.full((M, 256), top, device="cuda").bfloat16()
        y = b.nvfp4_gemv(x, W, b.DT_F32).double()
        want = top * 2.0 ** -30 * 256
        assert float((y / want - 1).abs().max()) <= 2.0 ** -15
