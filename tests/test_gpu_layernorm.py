"""Layer norm against float64.

Tolerances, from the sums' lengths: a sum over D <= 16384 elements is at most 64 additions deep (32 in a thread, 5 + 15 across, a product each), so it
is off by 2^-18 of the sum of magnitudes; mean, 1 / sqrt(...) and xh = (x - m) r inherit that: xh is off by 2^-18 (r mean|x| + |xh|). The sums over
rows are at most 128 additions deep for T <= 16384 (rows of a group, groups, CTAs): 2^-16 of the sum of magnitudes. Roundings to the output types come on top."""
import numpy as np
import pytest
import torch

from oracle import block_ops as O
from paper_2510_27527_b200 import synth
from tests.block_util import BF16, F32, device_rows, guarded, host, inputs, untouched

pytestmark = pytest.mark.gpu
DEEP = 2.0 ** -18


def params(D, dtype, seed=9):
    rng = np.random.default_rng(seed)
    g, b = (1 + 0.2 * rng.standard_normal(D)).astype(np.float32), (0.3 * rng.standard_normal(D)).astype(np.float32)
    if dtype == torch.bfloat16:
        g, b = synth.round_to_bf16(g), synth.round_to_bf16(b)
    return g, b, torch.from_numpy(g).cuda().to(dtype), torch.from_numpy(b).cuda().to(dtype)


def check(name, got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300))))


def run(T, D, x_dtype, p_dtype, save, has_beta=True, x=None, eps=1e-5, offset=0.5):
    from paper_2510_27527_b200 import binding as b

    x = inputs(T, D, T + D, x_dtype) + np.float32(offset) if x is None else x
    if x_dtype == torch.bfloat16:
        x = synth.round_to_bf16(x)
    gamma, beta, G, B = params(D, p_dtype)
    dy = synth.gradients(T, D, 5, 1e-3)
    X, dY = device_rows(x, x_dtype), device_rows(dy, torch.bfloat16)
    view, buf = guarded(T, D, torch.bfloat16)
    Y, saved = b.nvfp4_layernorm_fwd(X, G, B if has_beta else None, eps, save, out=view)
    assert untouched(view, buf)
    x64, g64, dy64 = x.astype(np.float64), gamma.astype(np.float64), dy.astype(np.float64)
    y, mean, r = O.layernorm(x64, g64, beta.astype(np.float64) if has_beta else None, eps)
    xh = (x64 - mean) * r
    axh = r * np.abs(x64).mean(1, keepdims=True) + np.abs(xh)
    check("y", host(Y), y, BF16 * np.abs(y) + DEEP * np.abs(g64) * axh + 2 * F32 * np.abs(beta) + 1e-38)
    if save == 0:
        assert saved is None
        return
    if save == 2:
        codes, scales, x64 = O.ckpt8(x)
        assert np.array_equal(saved.x8.codes.cpu().numpy(), codes) and np.array_equal(saved.x8.scales.cpu().numpy(), scales)
        X.fill_(float("nan"))  # backward must not need it
        xh = (x64 - mean) * r
        axh = r * np.abs(x64).mean(1, keepdims=True) + np.abs(xh) + r * np.abs(mean)
    dx, dg, db = O.layernorm_bwd(dy64, x64, mean, r, g64)
    view, buf = guarded(T, D, x_dtype)
    dX, dG, dB = b.nvfp4_layernorm_bwd(dY, saved, view)
    assert untouched(view, buf) and (dB is not None) == has_beta
    h = dy64 * g64
    c2 = (h * xh).mean(1, keepdims=True)
    err = DEEP * (np.abs(h) + np.abs(h).mean(1, keepdims=True) + np.abs(xh) * (np.abs(h * xh).mean(1, keepdims=True) + (np.abs(h) * axh).mean(1, keepdims=True)) + np.abs(c2) * axh)
    check("dx", host(dX), dx, (BF16 if x_dtype == torch.bfloat16 else F32) * np.abs(dx) + DEEP * np.abs(dx) + r * err + 1e-38)
    last = BF16 if p_dtype == torch.bfloat16 else F32
    check("dgamma", host(dG), dg, last * np.abs(dg) + 2.0 ** -16 * np.abs(dy64 * xh).sum(0) + DEEP * (np.abs(dy64) * axh).sum(0) + 1e-38)
    if has_beta:
        check("dbeta", host(dB), db, last * np.abs(db) + 2.0 ** -16 * np.abs(dy64).sum(0) + 1e-38)


@pytest.mark.parametrize("save", [0, 1, 2])
@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D", [(1, 1), (1, 8), (3, 33), (2, 255), (9, 256), (17, 264), (5, 500), (8, 513), (31, 768), (3, 1000), (64, 1024), (7, 1025), (4, 1416), (5, 1600),
                                 (6, 2048), (3, 2816), (2, 3500), (9, 4096), (3, 5120), (2, 7000), (4, 8192), (2, 10001), (3, 16384)])
def test_forward_and_backward(T, D, x_dtype, save):
    run(T, D, x_dtype, torch.float32 if (T + save) % 2 else torch.bfloat16, save)


@pytest.mark.parametrize("T,D", [(5000, 64), (2000, 1024), (1201, 1500), (777, 4000), (700, 8192), (650, 9000)])
@pytest.mark.parametrize("save", [1, 2])
def test_many_rows(T, D, save):
    run(T, D, torch.bfloat16, torch.float32, save, has_beta=save == 2)


def test_rows_that_hardly_vary():
    """Mean far larger than the spread, constant rows, tiny and large values."""
    D = 1000
    x = inputs(6, D, 3, torch.float32, hot=False)
    x[0] += 1000
    x[1] = 3.25
    x[2] = 0
    x[3] *= 1e-18
    x[4] *= 1e15
    run(6, D, torch.float32, torch.float32, 1, x=x.astype(np.float32))
    run(6, D, torch.float32, torch.float32, 2, x=x.astype(np.float32))


def test_gradients_agree_with_differences():
    """The kernels' own forward, in FP32 rows: the loss is summed in float64 over BF16 results, so steps are large and the bound is loose."""
    from paper_2510_27527_b200 import binding as b

    T, D = 4, 64
    x, dy = inputs(T, D, 1, torch.float32, hot=False), synth.gradients(T, D, 2, 1.0)
    _, _, G, B = params(D, torch.float32)
    X, dY = torch.from_numpy(x).cuda(), b.upload_bf16(dy)
    _, saved = b.nvfp4_layernorm_fwd(X, G, B)
    dX, dG, dB = b.nvfp4_layernorm_bwd(dY, saved)
    rng = np.random.default_rng(0)
    for _ in range(5):
        d = torch.from_numpy(rng.standard_normal((T, D)).astype(np.float32)).cuda()
        step = 0.05
        up, down = (float((b.nvfp4_layernorm_fwd(X + s * step * d, G, B)[0].double() * dY.double()).sum()) for s in (1, -1))
        want = float((dX.double() * d.double()).sum())
        y = b.nvfp4_layernorm_fwd(X, G, B)[0].double()
        # roundings of the two results to BF16, each 2^-8 |y dy| at most, and the difference's third-order term
        room = 2 * BF16 * float((y.abs() * dY.double().abs()).sum()) / (2 * step) * 1.2 + step ** 2 * 10 * float(dX.double().abs().sum())
        assert abs((up - down) / (2 * step) - want) <= room


def test_nothing_to_do():
    from paper_2510_27527_b200 import binding as b

    _, _, G, B = params(40, torch.float32)
    e = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda")
    for save in (0, 1, 2):
        Y, saved = b.nvfp4_layernorm_fwd(e, G, B, save=save)
        assert Y.shape == (0, 40)
        if save:
            dX, dG, dB = b.nvfp4_layernorm_bwd(e, saved)
            assert dX.shape == (0, 40) and not dG.any() and not dB.any()


def test_not_finite_rows_spoil_no_other():
    from paper_2510_27527_b200 import binding as b

    x = inputs(40, 300, 2)
    _, _, G, B = params(300, torch.bfloat16)
    good = b.nvfp4_layernorm_fwd(device_rows(x, torch.bfloat16), G, B)[0]
    x[7, 5], x[8, 299] = np.nan, np.inf
    y, saved = b.nvfp4_layernorm_fwd(device_rows(x, torch.bfloat16), G, B, save=2)
    rest = [i for i in range(40) if i not in (7, 8)]
    assert torch.isnan(y[7]).all() and torch.isnan(y[8]).all() and torch.equal(y[rest], good[rest])
    dX, _, _ = b.nvfp4_layernorm_bwd(device_rows(synth.gradients(40, 300, 1), torch.bfloat16), saved)
    assert torch.isnan(dX[7:9]).all() and torch.isfinite(dX[rest]).all()


def test_in_place_repeated_and_captured():
    from paper_2510_27527_b200 import binding as b

    T, D = 300, 1000
    X, dY = device_rows(inputs(T, D, 1), torch.bfloat16), device_rows(synth.gradients(T, D, 2), torch.bfloat16)
    _, _, G, B = params(D, torch.float32)
    Y, saved = b.nvfp4_layernorm_fwd(X, G, B, save=2)
    want = b.nvfp4_layernorm_bwd(dY, saved)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(b.nvfp4_layernorm_bwd(dY, saved), want))  # fixed orders
    d = dY.clone()
    assert torch.equal(b.nvfp4_layernorm_bwd(d, saved, dX=d)[0], want[0])
    graphs, outs = [], []
    for _ in range(2):  # two graphs, each with workspaces of its own, replayed side by side
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y, s = b.nvfp4_layernorm_fwd(X, G, B, save=2)
            outs.append((y, *b.nvfp4_layernorm_bwd(dY, s)))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(p, q) for p, q in zip(o, (Y, *want)))
