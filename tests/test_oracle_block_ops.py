"""Pins of the float64 definitions of the steps around the linears: formats against torch's casts, gradients against differences."""
import numpy as np
import pytest
import torch

from oracle import block_ops as O
from paper_2510_27527_b200 import synth


def test_e4m3_values_are_torchs():
    codes = torch.arange(127, dtype=torch.uint8)
    assert np.array_equal(O.e4m3_magnitudes(), codes.view(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("scale", [1e-38, 1e-20, 1.0, 3e37])
def test_checkpoint_codes_are_the_nearest_values(scale):
    rng = np.random.default_rng(1)
    x = synth.round_to_bf16((rng.standard_t(2, size=(40, 77)) * scale).clip(-3.3e38, 3.3e38).astype(np.float32))
    codes, scales, values = O.ckpt8(x)
    wide = np.zeros((40, 96), dtype=np.float64)
    wide[:, :77] = x
    y = torch.from_numpy(wide / np.ldexp(1.0, scales.astype(int) - 127).repeat(32, 1))
    assert np.array_equal(codes, y.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert y.abs().max() <= 448
    assert np.array_equal(values, (torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy() * np.ldexp(1.0, scales.astype(int) - 127).repeat(32, 1))[:, :77])


def test_checkpoint_edges():
    x = np.zeros((6, 32))
    x[1, 3], x[2, :2], x[3, :2], x[4, 0], x[5, 0] = 448.0, (449.0, 1.0), (np.inf, 2.0), np.nan, -0.0
    codes, scales, values = O.ckpt8(x)
    assert list(scales[:, 0]) == [10, 127, 128, 120, 10, 10]  # empty, exactly 448, above it, 2 = 256 * 2^-7 beside an infinity, NaN, -0
    assert values[1, 3] == 448 and values[2, 0] == 448 and values[3, 1] == 2 and np.isnan(values[3, 0]) and np.isnan(values[4, 0])
    assert codes[5, 0] == 0x80 and codes[3, 0] == 0x7F


def test_gradients_agree_with_differences():
    rng = np.random.default_rng(2)
    x, gamma, beta, dy = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    loss = lambda x, g, b: (O.layernorm(x, g, b, 1e-3)[0] * dy).sum()  # noqa: E731
    _, mean, r = O.layernorm(x, gamma, beta, 1e-3)
    u = rng.standard_normal((3, 7))
    loss2 = lambda g, u: (O.swiglu(g, u) * dy).sum()  # noqa: E731
    for f, at, grads in ((loss, (x, gamma, beta), O.layernorm_bwd(dy, x, mean, r, gamma)), (loss2, (x, u), O.swiglu_bwd(dy, x, u))):
        for k, (a, grad) in enumerate(zip(at, grads)):
            for i in np.ndindex(a.shape):
                d = np.zeros_like(a)
                d[i] = 1e-6
                up, down = [f(*(v + s * d if j == k else v for j, v in enumerate(at))) for s in (1, -1)]
                assert abs((up - down) / 2e-6 - grad[i]) <= 1e-7 * (1 + abs(grad[i]))
