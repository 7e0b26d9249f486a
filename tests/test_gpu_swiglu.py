"""SwiGLU against float64.

Tolerances: exp is off by 2 + 1.173 |g| units of 2^-23, the sum and the quotient by 3 more, so the sigmoid s by eps = (6 + 1.2 |g|) 2^-23 of itself;
products add 2^-24 each and the result's rounding 2^-8. In s (1 + g (1 - s)) the inner difference is off by s eps + 2^-24. The sigmoid is 0
where it is below 2^-126: 2^-126 of the products is allowed everywhere, and BF16's smallest number."""
import numpy as np
import pytest
import torch

from oracle import block_ops as O
from paper_2510_27527_b200 import synth
from tests.block_util import BF16, device_rows, guarded, host, inputs, untouched

pytestmark = pytest.mark.gpu
SIZES = [(1, 1), (1, 8), (2, 31), (3, 40), (5, 33), (77, 2816), (130, 1000), (64, 257)]


def tolerances(dh, g, u, h, dg, du):
    eps = (10 + 1.2 * np.abs(g)) * 2.0 ** -23
    s = O._sigmoid(g)
    floor = 2.0 ** -126 * (1 + np.abs(u)) * (1 + np.abs(g)) * 4 + 2.0 ** -133
    th = BF16 * np.abs(h) + eps * np.abs(h) + floor
    if dh is None:
        return th
    tdu = BF16 * np.abs(du) + eps * np.abs(du) + floor * np.abs(dh)
    # each factor's error, and that of 1 - s inside
    tdg = BF16 * np.abs(dg) + np.abs(dh * u) * s * (2 * eps * (1 + np.abs(g * O._sigmoid(-g))) + np.abs(g) * (s * eps + 2.0 ** -23)) + floor * np.abs(dh)
    return th, tdg + 2.0 ** -133, tdu + 2.0 ** -133


@pytest.mark.parametrize("save", [0, 1, 2])
@pytest.mark.parametrize("T,D", SIZES)
def test_forward_and_backward(T, D, save):
    from paper_2510_27527_b200 import binding as b

    g, u, dh = inputs(T, D, 1) * 1.0, inputs(T, D, 2), synth.gradients(T, D, 3, 1e-3)
    G, U, dH = (device_rows(v, torch.bfloat16) for v in (g, u, dh))
    view, buf = guarded(T, D, torch.bfloat16)
    H, saved = b.nvfp4_swiglu_fwd(G, U, save, out=view)
    assert H is view and untouched(view, buf)
    g64, u64 = g.astype(np.float64), u.astype(np.float64)
    h = O.swiglu(g64, u64)
    assert np.all(np.abs(host(H) - h) <= tolerances(None, g64, u64, h, None, None))
    if save == 0:
        assert saved is None
        return
    if save == 2:
        for ck, v in ((saved.g8, g), (saved.u8, u)):
            codes, scales, values = O.ckpt8(v)
            assert np.array_equal(ck.codes.cpu().numpy(), codes) and np.array_equal(ck.scales.cpu().numpy(), scales)
        G.fill_(float("nan")), U.fill_(float("nan"))  # backward must not need them
        g64, u64 = O.ckpt8(g)[2], O.ckpt8(u)[2]
    (vg, bg), (vu, bu) = guarded(T, D, torch.bfloat16), guarded(T, D, torch.bfloat16, extra_cols=0)
    b.nvfp4_swiglu_bwd(dH, saved, vg, vu)
    dh64 = dh.astype(np.float64)
    dg, du = O.swiglu_bwd(dh64, g64, u64)
    _, tg, tu = tolerances(dh64, g64, u64, O.swiglu(g64, u64), dg, du)
    assert np.all(np.abs(host(vg) - dg) <= tg) and np.all(np.abs(host(vu) - du) <= tu)
    assert untouched(vg, bg) and untouched(vu, bu)


def test_large_and_infinite_gates():
    from paper_2510_27527_b200 import binding as b

    g = np.array([[-3e38, -1000, -100, -88.5, -87, -50, -20, -1e-30, 0, 1e-30, 20, 50, 88, 100, 1000, 3e38]], dtype=np.float32)
    g = synth.round_to_bf16(g)
    u = np.full_like(g, 0.75)
    H, saved = b.nvfp4_swiglu_fwd(device_rows(g, torch.bfloat16), device_rows(u, torch.bfloat16))
    g64, u64 = g.astype(np.float64), u.astype(np.float64)
    h = O.swiglu(g64, u64)
    assert np.all(np.abs(host(H) - h) <= tolerances(None, g64, u64, h, None, None))
    dG, dU = b.nvfp4_swiglu_bwd(device_rows(np.ones_like(g), torch.bfloat16), saved)
    dg, du = O.swiglu_bwd(np.ones_like(g64), g64, u64)
    _, tg, tu = tolerances(np.ones_like(g64), g64, u64, h, dg, du)
    assert np.all(np.abs(host(dG) - dg) <= tg) and np.all(np.abs(host(dU) - du) <= tu)
    x = torch.tensor([[float("nan"), float("-inf"), 1.0, float("inf")]], dtype=torch.bfloat16, device="cuda")
    H, _ = b.nvfp4_swiglu_fwd(x, torch.ones_like(x))
    assert torch.isnan(H[0, :2]).all() and torch.isfinite(H[0, 2]) and H[0, 3] == float("inf")


def test_in_place_and_the_same_tensor_twice():
    from paper_2510_27527_b200 import binding as b

    T, D = 50, 200
    g, u, dh = (device_rows(inputs(T, D, i), torch.bfloat16) for i in (1, 2, 3))
    want, saved = b.nvfp4_swiglu_fwd(g, u, 2)
    wg, wu = b.nvfp4_swiglu_bwd(dh, saved)
    for target in (0, 1):
        pair = [g.clone(), u.clone()]
        H, _ = b.nvfp4_swiglu_fwd(*pair, 0, out=pair[target])
        assert torch.equal(H, want)
    d = dh.clone()
    dG, dU = b.nvfp4_swiglu_bwd(d, saved, dG=d)
    assert torch.equal(dG, wg) and torch.equal(dU, wu)
    H, _ = b.nvfp4_swiglu_fwd(g, g)
    assert torch.equal(H, b.nvfp4_swiglu_fwd(g, g.clone())[0])


@pytest.mark.parametrize("save", [1, 2])
@pytest.mark.parametrize("T,D", [(1, 32), (5, 96), (300, 2816), (77, 40)])
def test_without_gaps(T, D, save):
    """Matrices whose rows follow one another give what the same rows in wider buffers give."""
    from paper_2510_27527_b200 import binding as b

    wide = [device_rows(v, torch.bfloat16) for v in (inputs(T, D, 1), inputs(T, D, 2), synth.gradients(T, D, 3, 1e-3))]
    flat = [v.contiguous() for v in wide]
    H, saved = b.nvfp4_swiglu_fwd(flat[0], flat[1], save)
    H2, saved2 = b.nvfp4_swiglu_fwd(wide[0], wide[1], save)
    assert torch.equal(H, H2)
    if save == 2:
        assert torch.equal(saved.g8.buf, saved2.g8.buf) and torch.equal(saved.u8.buf, saved2.u8.buf)
    assert all(torch.equal(p, q) for p, q in zip(b.nvfp4_swiglu_bwd(flat[2], saved), b.nvfp4_swiglu_bwd(wide[2], saved2)))


def test_no_rows():
    from paper_2510_27527_b200 import binding as b

    e = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda")
    for save in (0, 1, 2):
        H, saved = b.nvfp4_swiglu_fwd(e, e, save)
        assert H.shape == (0, 40)
        if save:
            assert b.nvfp4_swiglu_bwd(e, saved)[0].shape == (0, 40)
