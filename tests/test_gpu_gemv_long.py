"""nvfp4_gemv where a CTA goes around its ring of stages, brings X behind the first weights and stages X in pieces, against float64.

Operands are made of random codes and scale bytes, so that their values are known without a quantizer. Tolerance as in test_gpu_gemv.py: an instruction
adds 16 products and a sum at 24 bits, 17 * 2^-23; eight of them a piece of 128; a warp adds half of its CTA's pieces, 64 in the longest case here, and
then ten partial sums, at 2^-24 each: 136 * 2^-23 + 74 * 2^-24 < 2^-15 of sum |x w|."""
import pytest
import torch

from tests.block_util import BF16

pytestmark = pytest.mark.gpu
E2M1 = [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]


def operand(N, K, gs, seed=1):
    """(operand, its values in float64 [N, K])."""
    from paper_2510_27527_b200 import binding as b

    g = torch.Generator(device="cuda").manual_seed(seed)
    Kp = (K + 127) // 128 * 128
    nb, nbp = Kp // 16, (Kp // 16 + 15) // 16 * 16
    codes = torch.randint(0, 16, (N, Kp), generator=g, device="cuda", dtype=torch.uint8)
    codes[:, K:] = 0
    scales = torch.randint(40, 88, (N, nb), generator=g, device="cuda", dtype=torch.uint8)  # E4M3 bytes of 2^-2 .. 15
    r, kb = torch.arange(N, device="cuda")[:, None], torch.arange(nb, device="cuda")[None]
    sf = torch.full(((N + 127) // 128 * 128 * nbp,), 0x7F, dtype=torch.uint8, device="cuda")  # NaN where no block is
    sf[((r >> 7) * (nbp >> 2) + (kb >> 2)) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4 + (kb & 3)] = scales
    gscale = torch.rand({0: 1, 1: N, 2: N * (Kp // 128)}[gs], generator=g, device="cuda") * 1e-3 + 1e-4
    wide = {0: lambda: gscale.view(1, 1), 1: lambda: gscale.view(N, 1), 2: lambda: gscale.view(N, -1).repeat_interleave(8, 1)}[gs]().double()
    values = torch.tensor(E2M1, dtype=torch.float64, device="cuda")[codes.int()]
    values.view(N, nb, 16).mul_((scales.view(torch.float8_e4m3fn).double() * wide)[..., None])
    return b.Operand((codes[:, 0::2] | codes[:, 1::2] << 4).reshape(-1).contiguous(), sf, gscale, N, K, gs, b.SF_TILED128x4), values[:, :K]


def tokens(M, K, seed=2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, K, generator=g, device="cuda")
    x[:, torch.randperm(K, generator=g, device="cuda")[: K // 50]] *= 30
    buf = torch.full((M, (K + 7) // 8 * 8 + 8), float("nan"), device="cuda").bfloat16()
    buf[:, :K] = x
    return buf[:, :K]


def check(y, x, w, more=0.0, f32=True):
    want, absdot = x.double() @ w.T + more, x.double().abs() @ w.abs().T + (more.abs() if isinstance(more, torch.Tensor) else 0.0)
    bad = ~((y.double() - want).abs() <= 2.0 ** -15 * absdot + (0.0 if f32 else BF16) * want.abs())
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:5].tolist())


@pytest.mark.parametrize("gs", [0, 1, 2])
@pytest.mark.parametrize("M,N,K", [(1, 128, 20000), (2, 100, 20001), (3, 130, 20000), (4, 128, 30000), (5, 128, 20000), (9, 300, 9000), (16, 128, 20111), (32, 128, 20000), (33, 70, 20000),
                                   (1, 4100, 8192), (4, 4100, 8192), (16, 7000, 4096), (20, 7000, 4096)])
def test_several_times_around_the_ring(M, N, K, gs):
    from paper_2510_27527_b200 import binding as b

    W, w = operand(N, K, gs)
    x = tokens(M, K)
    check(b.nvfp4_gemv(x, W, b.DT_F32), x, w)
    check(b.nvfp4_gemv(x, W), x, w, f32=False)


@pytest.mark.parametrize("gs", [0, 2])
@pytest.mark.parametrize("M,N,K", [(2, 19200, 8192), (1, 19200, 16384), (2, 19200, 16384), (4, 19200, 4096), (7, 19200, 4096), (32, 19200, 2048), (1, 37900, 2048), (2, 38100, 2048)])
def test_more_row_tiles_than_are_split(M, N, K, gs):
    """One CTA takes all of k: X of one and two tokens is staged in pieces where they are more than it holds."""
    from paper_2510_27527_b200 import binding as b

    W, w = operand(N, K, gs)
    x = tokens(M, K)
    y = b.nvfp4_gemv(x, W, b.DT_F32)
    check(y, x, w)
    if M == 2:
        assert torch.equal(b.nvfp4_gemv(x[1:], W, b.DT_F32), y[1:])


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 16, 32])
@pytest.mark.parametrize("N,D,n_out", [(128, 20300, 300), (150, 20000, 65), (150, 600, 64), (19000, 2100, 700)])
def test_outlier_channels_after_the_codes(M, N, D, n_out):
    """Their steps are the last of the ring, in every form of the kernel, also where a CTA has nothing else."""
    from paper_2510_27527_b200 import binding as b

    g = torch.Generator(device="cuda").manual_seed(3)
    order = torch.randperm(D, generator=g, device="cuda")
    outl, keep = order[:n_out].sort().values, order[n_out:].sort().values
    W, w = operand(N, D - n_out, 2)
    Kh = b.lib.nvfp4_outlier_pad(n_out)
    wo = torch.zeros(N, Kh, device="cuda").bfloat16()
    wo[:, :n_out] = torch.randn(N, n_out, generator=g, device="cuda") * 0.02
    bias = torch.randn(N, generator=g, device="cuda").bfloat16()
    x = tokens(M, D)
    x[:, outl] *= 32
    y = b.nvfp4_gemv(x, W, b.DT_F32, bias=bias, index=(outl.int(), keep.int()), W_out=wo)
    whole = torch.zeros(N, D, dtype=torch.float64, device="cuda")
    whole[:, keep], whole[:, outl] = w, wo[:, :n_out].double()
    check(y, x, whole, bias.double())


@pytest.mark.parametrize("M", [1, 2, 4, 16, 32])
def test_repeated_calls_agree(M):
    """Fixed orders, whichever CTA is first."""
    from paper_2510_27527_b200 import binding as b

    W, _ = operand(1000, 20000, 1)
    x = tokens(M, 20000)
    want = b.nvfp4_gemv(x, W, b.DT_F32)
    assert all(torch.equal(b.nvfp4_gemv(x, W, b.DT_F32), want) for _ in range(20))
