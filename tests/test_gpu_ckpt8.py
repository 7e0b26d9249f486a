"""Activation checkpoints in 8 bits: codes, scales and values bit for bit."""
import numpy as np
import pytest
import torch

from oracle import block_ops as O
from paper_2510_27527_b200 import synth
from tests.block_util import device_rows, guarded, host, inputs, untouched

pytestmark = pytest.mark.gpu


def pack_and_compare(x: np.ndarray, dtype):
    from paper_2510_27527_b200 import binding as b

    R, K = x.shape
    ck = b.alloc_ckpt8(R, K)
    tail = torch.full((ck.buf.numel() + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    ck.buf = tail[:-64]
    b.nvfp4_ckpt8_pack(device_rows(x, dtype), ck)
    codes, scales, values = O.ckpt8(x)
    bad = np.argwhere(ck.codes.cpu().numpy() != codes)
    assert len(bad) == 0, (len(bad), bad[:5].tolist())
    assert np.array_equal(ck.scales.cpu().numpy(), scales)
    assert bool((tail[-64:] == 0xA5).all())
    for out, code in ((torch.bfloat16, b.DT_BF16), (torch.float32, b.DT_F32)):
        view, buf = guarded(R, K, out)
        b.nvfp4_ckpt8_unpack(ck, code, view)
        assert np.array_equal(host(view), values, equal_nan=True)
        assert untouched(view, buf)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,K", [(1, 1), (1, 7), (3, 8), (5, 31), (2, 32), (7, 33), (4, 100), (33, 257), (129, 1000), (300, 1024)])
def test_pack_and_unpack(R, K, dtype):
    pack_and_compare(inputs(R, K, R + K, dtype), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,K", [(1, 32), (3, 64), (257, 96), (700, 1024), (3000, 2048)])
def test_without_gaps(R, K, dtype):
    """Matrices whose rows follow one another give what the same rows in a wider buffer give."""
    from paper_2510_27527_b200 import binding as b

    x = torch.from_numpy(inputs(R, K, 1, dtype)).cuda().to(dtype)
    wide = torch.full((R, K + 16), float("nan"), dtype=dtype, device="cuda")
    wide[:, :K] = x
    ck, other = b.nvfp4_ckpt8_pack(x), b.nvfp4_ckpt8_pack(wide[:, :K])
    assert torch.equal(ck.buf, other.buf)
    if R * K <= 100000:
        codes, scales, _ = O.ckpt8(host(x))
        assert np.array_equal(ck.codes.cpu().numpy(), codes) and np.array_equal(ck.scales.cpu().numpy(), scales)
    for out, code in ((torch.bfloat16, b.DT_BF16), (torch.float32, b.DT_F32)):
        view, buf = guarded(R, K, out)
        assert torch.equal(b.nvfp4_ckpt8_unpack(ck, code), b.nvfp4_ckpt8_unpack(ck, code, view)) and untouched(view, buf)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [1e-39, 1e-36, 1e-30, 1e30, 1e37])
def test_scales_at_the_ends_of_the_range(scale, dtype):
    x = inputs(9, 70, 1, torch.bfloat16, hot=False) * np.float64(scale)
    x = x.astype(np.float32)
    pack_and_compare(x if dtype == torch.float32 else synth.round_to_bf16(x), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_border_of_the_format(dtype):
    """All ties between neighbouring codes, in both types, under scales from group maxima at and beside 448 * 2^e."""
    table = O.e4m3_magnitudes()
    mid = (table[1:] + table[:-1]) / 2
    v = np.concatenate([table, mid, -mid, [0.0, -0.0, 2.0 ** -11, -2.0 ** -11, 2.0 ** -12]])
    rows = []
    for top in (448.0, 446.0, 450.0, 224.0, 1.0, 255.0):
        vs = v[np.abs(v) <= top]
        vs = np.resize(vs, -(-len(vs) // 31) * 31).reshape(-1, 31)
        rows.append(np.concatenate([np.full((len(vs), 1), top), vs], 1))
    x = np.concatenate(rows).astype(np.float32)
    if dtype == torch.bfloat16:
        x = synth.round_to_bf16(x)
    pack_and_compare(x, dtype)
    pack_and_compare((x * np.float32(2.0 ** -30)).astype(np.float32), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_not_finite(dtype):
    x = inputs(6, 96, 4, torch.bfloat16)
    x[0, 3], x[1, 40], x[2, 95], x[3, :32], x[4, 0], x[5, 64:] = np.inf, -np.inf, np.nan, np.nan, -0.0, 0.0
    x[0, 32:64:2] = np.nan  # every other element
    x[1, :32], x[1, 5] = np.nan, 3.0
    pack_and_compare(x, dtype)


def test_nothing_to_do_and_refusals():
    from paper_2510_27527_b200 import binding as b

    ck = b.nvfp4_ckpt8_pack(torch.empty(0, 40, dtype=torch.bfloat16, device="cuda"))
    assert ck.buf.numel() == 0 and b.nvfp4_ckpt8_unpack(ck).shape == (0, 40)
    x = torch.ones(4, 40, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(RuntimeError, match="checkpoint"):
        b.nvfp4_ckpt8_pack(x, b.alloc_ckpt8(4, 48))
    with pytest.raises(b.Nvfp4Error):
        b.nvfp4_ckpt8_pack(torch.ones(4, 41, dtype=torch.bfloat16, device="cuda"))  # rows off their 16-byte boundaries
    with pytest.raises(RuntimeError, match="columns at a stride"):
        b.nvfp4_ckpt8_pack(torch.ones(40, 4, dtype=torch.bfloat16, device="cuda").T)


def test_large_offsets():
    """More than 2^31 elements: rows beyond the reach of 32 bits."""
    from paper_2510_27527_b200 import binding as b

    R, K = 270000, 8192
    x = torch.zeros(R, K, dtype=torch.bfloat16, device="cuda")
    part = torch.from_numpy(inputs(3, K, 1)).cuda().bfloat16()
    x[-3:] = part
    ck = b.nvfp4_ckpt8_pack(x)
    small = b.nvfp4_ckpt8_pack(part)
    assert torch.equal(ck.codes[-3:], small.codes) and torch.equal(ck.scales[-3:], small.scales)
    assert int(ck.codes[:-3].max()) == 0 and int(ck.scales[:-3].max()) == 10
    b.nvfp4_ckpt8_unpack(ck, out=x.fill_(5))
    assert torch.equal(x[-3:], b.nvfp4_ckpt8_unpack(small)) and not x[:-3].any()
