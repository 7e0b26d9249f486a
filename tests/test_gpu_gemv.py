"""nvfp4_gemv against float64 products of the dequantized weights.

Tolerance of an FP32 result, relative to a = sum_k |x_k w_k|: an instruction adds 16 products and a sum at 24 bits, cutting what lies below,
17 * 2^-23; 8 instructions a piece of 128, then at most 112 / 2 pieces and 10 partial sums at 2^-24 each: 136 * 2^-23 + 66 * 2^-24 < 2^-15. Elements
of X below 2^-28 of the largest in their 128 add 2^-39 of it each, nothing beside that. A result in BF16 is off by 2^-8 of itself more."""
import numpy as np
import pytest
import torch

from oracle import nvfp4_oracle as orc
from paper_2510_27527_b200 import synth
from tests.block_util import BF16, device_rows, guarded, host, untouched
from tests.gpu_util import upload_operand

pytestmark = pytest.mark.gpu


def weights(N, K, gs, seed=1):
    from paper_2510_27527_b200 import binding as b

    q = orc.quantize(synth.weights(N, K, seed), orc.AXIS_ROW, orc.RTN, gs, 0, 2)
    return upload_operand(q, b), orc.dequantize(q)[:, :K]


def check(y, want, absdot, f32):
    tol = 2.0 ** -15 * absdot + (0 if f32 else BF16 * np.abs(want)) + 1e-30
    bad = np.abs(y - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), float(np.abs(y - want).max()))


@pytest.mark.parametrize("gs", [0, 1, 2])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 40, 16), (1, 64, 128), (2, 17, 100), (3, 65, 129), (4, 300, 700), (3, 2100, 5000), (4, 4000, 2816), (5, 129, 900), (8, 130, 1000), (9, 16, 257), (15, 200, 384), (16, 128, 1416),
                                   (17, 333, 640), (31, 96, 260), (32, 1024, 1024), (33, 100, 1001), (70, 48, 2816)])
def test_against_float64(M, N, K, gs):
    from paper_2510_27527_b200 import binding as b

    W, w = weights(N, K, gs)
    x, _ = synth.activations(M, K, 3, n_outlier=max(1, K // 50), factor=30.0)
    X = device_rows(x, torch.bfloat16)
    want, absdot = x.astype(np.float64) @ w.T, np.abs(x).astype(np.float64) @ np.abs(w).T
    for dt, f32 in ((torch.float32, True), (torch.bfloat16, False)):
        view, buf = guarded(M, N, dt, extra_cols=16)
        b.nvfp4_gemv(X, W, b.DT_F32 if f32 else b.DT_BF16, out=view)
        check(host(view), want, absdot, f32)
        assert untouched(view, buf)


@pytest.mark.parametrize("M", [1, 5, 32])
@pytest.mark.parametrize("D,n_out", [(200, 1), (257, 63), (1024, 102), (130, 66)])
def test_outlier_channels_and_bias(D, n_out, M):
    from paper_2510_27527_b200 import binding as b

    N = 150
    w_full = synth.weights(N, D, 5)
    outl = synth.outlier_channels(D, n_out, 7)
    keep = np.setdiff1d(np.arange(D), outl)
    q = orc.quantize(w_full[:, keep], orc.AXIS_ROW, orc.RTN, 2, 0, 2)
    Kh = b.lib.nvfp4_outlier_pad(n_out)
    wo = np.zeros((N, Kh), dtype=np.float32)
    wo[:, :n_out] = w_full[:, outl]
    bias = synth.round_to_bf16(np.random.default_rng(1).standard_normal(N).astype(np.float32))
    x, _ = synth.activations(M, D, 3)
    x[:, outl] *= 32
    index = (torch.from_numpy(outl.astype(np.int32)).cuda(), torch.from_numpy(keep.astype(np.int32)).cuda())
    y = b.nvfp4_gemv(device_rows(x, torch.bfloat16), upload_operand(q, b), b.DT_F32, bias=b.upload_bf16(bias), index=index, W_out=b.upload_bf16(wo))
    w = np.zeros((N, D))
    w[:, keep], w[:, outl] = orc.dequantize(q)[:, : len(keep)], w_full[:, outl]
    check(host(y), x.astype(np.float64) @ w.T + bias, np.abs(x).astype(np.float64) @ np.abs(w).T + np.abs(bias), True)


def test_a_tokens_result_is_its_own():
    """The order of a token's sums does not depend on the others (from five tokens on, for three and four, and for one and two), and a non-finite token spoils no
    other."""
    from paper_2510_27527_b200 import binding as b

    W, _ = weights(300, 1500, 2)
    x, _ = synth.activations(40, 1500, 3)
    X = device_rows(x, torch.bfloat16)
    whole = b.nvfp4_gemv(X, W, b.DT_F32)
    assert torch.equal(b.nvfp4_gemv(X[2:7], W, b.DT_F32), whole[2:7]) and torch.equal(b.nvfp4_gemv(X[30:38], W, b.DT_F32), whole[30:38])
    for m in (0, 7, 8, 20, 36):
        one = b.nvfp4_gemv(X[m: m + 1], W, b.DT_F32)
        assert torch.equal(b.nvfp4_gemv(X[m: m + 2], W, b.DT_F32)[:1], one)
        assert torch.equal(b.nvfp4_gemv(X[m: m + 4], W, b.DT_F32)[:3], b.nvfp4_gemv(X[m: m + 3], W, b.DT_F32))
        assert torch.allclose(one, whole[m: m + 1], rtol=1e-4, atol=1e-4)
    assert torch.equal(b.nvfp4_gemv(X[3:14], W, b.DT_F32), whole[3:14])
    X[5, 77], X[6, 1499] = float("inf"), float("nan")
    y = b.nvfp4_gemv(X, W, b.DT_F32)
    assert not torch.isfinite(y[5]).any() and torch.isnan(y[6]).all()
    rest = [i for i in range(40) if i not in (5, 6)]
    assert torch.equal(y[rest], whole[rest])


def test_wide_ranges_within_a_token():
    """Values far apart: FP16 in between must not show."""
    from paper_2510_27527_b200 import binding as b

    W, w = weights(64, 512, 0)
    rng = np.random.default_rng(0)
    x = synth.round_to_bf16((rng.standard_normal((6, 512)) * np.exp2(rng.uniform(-22, 0, (6, 512)))).astype(np.float32))
    x[1] *= np.float32(2.0 ** 100)
    x[2] *= np.float32(2.0 ** -100)
    x[3, 128:] *= np.float32(2.0 ** -60)  # a piece of its own scale
    x[4] = 0
    x[5, :] = np.float32(2.0 ** -126)
    want, absdot = x.astype(np.float64) @ w.T, np.abs(x).astype(np.float64) @ np.abs(w).T
    check(host(b.nvfp4_gemv(b.upload_bf16(x), W, b.DT_F32)), want, absdot, True)


def test_columns_that_x_does_not_have_are_nan():
    from paper_2510_27527_b200 import binding as b

    W, _ = weights(32, 60, 0)
    x = torch.ones(2, 64, dtype=torch.bfloat16, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    wo = torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda")
    for outl, keep in (([1, 2, 3, 64], list(range(60))), ([60, 61, 62, 63], [-1] + list(range(1, 60))), ([60, 61, 62, 2 ** 31 - 1], list(range(60)))):
        assert torch.isnan(b.nvfp4_gemv(x, W, b.DT_F32, index=(i32(outl), i32(keep)), W_out=wo)).all()


def test_no_tokens_and_no_rows():
    from paper_2510_27527_b200 import binding as b

    W, _ = weights(48, 64, 0)
    assert b.nvfp4_gemv(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), W).shape == (0, 48)
    one = torch.ones(1, 64, dtype=torch.bfloat16, device="cuda").expand(4, 64)  # a row that stands for several
    with pytest.raises(b.Nvfp4Error):
        b.nvfp4_gemv(one, W)
    with pytest.raises(RuntimeError, match="stride"):
        b.nvfp4_gemv(torch.ones(64, 4, dtype=torch.bfloat16, device="cuda").T, W)
    with pytest.raises(b.Nvfp4Error):
        b.nvfp4_gemv(torch.ones(2, 72, dtype=torch.bfloat16, device="cuda"), W)
    with pytest.raises(RuntimeError, match="too small"):
        b.nvfp4_gemv(torch.ones(2, 64, dtype=torch.bfloat16, device="cuda"), b.Operand(W.codes[:-1], W.sf, W.gscale, 48, 64, 0, 1))


def test_captured_and_on_another_stream():
    from paper_2510_27527_b200 import binding as b

    W, w = weights(500, 700, 1)
    x, _ = synth.activations(4, 704, 3)
    X = b.upload_bf16(x)[:, :700]
    want = b.nvfp4_gemv(X, W, b.DT_F32)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = b.nvfp4_gemv(X, W, b.DT_F32)
    s.synchronize()
    assert torch.equal(got, want)
    y = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.nvfp4_gemv(X, W, b.DT_F32, out=y)
    X.mul_(2)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, b.nvfp4_gemv(X, W, b.DT_F32)) and not torch.equal(y, want)
