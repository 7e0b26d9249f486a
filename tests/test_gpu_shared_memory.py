"""Results in the memory of inputs: what is allowed, and what the binding refuses."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def mk(*shape):
    return torch.randn(*shape, device="cuda").bfloat16()


def test_a_product_in_its_inputs_memory_is_refused():
    from paper_2510_27527_b200 import binding as b

    W, buf = b.nvfp4_quantize(mk(64, 64)), mk(5, 128)
    x = mk(4, 64)
    for X, Y in ((x, x), (buf[:4, :64], buf[:4, :64]), (buf.view(-1)[:256].view(4, 64), buf.view(-1)[64:320].view(4, 64))):
        with pytest.raises(RuntimeError, match="share memory"):
            b.nvfp4_gemv(X, W, out=Y)
    want = b.nvfp4_gemv(buf[:4, :64], W)
    b.nvfp4_gemv(buf[:4, :64], W, out=buf[:4, 64:])  # rows of one buffer, columns apart
    assert torch.equal(buf[:4, 64:], want)


def test_two_gradients_in_one_memory_are_refused():
    from paper_2510_27527_b200 import binding as b

    g, u, dh = mk(8, 64), mk(8, 64), mk(8, 64)
    _, saved = b.nvfp4_swiglu_fwd(g, u)
    want = b.nvfp4_swiglu_bwd(dh, saved)
    for o in (mk(8, 64), mk(8, 72)[:, :64]):
        with pytest.raises(RuntimeError, match="share memory"):
            b.nvfp4_swiglu_bwd(dh, saved, o, o)
    got = b.nvfp4_swiglu_bwd(dh, saved, g, u)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("save", [0, 2])
@pytest.mark.parametrize("T,D", [(3, 64), (700, 1000), (40, 9000)])
def test_a_norm_in_place(T, D, save):
    from paper_2510_27527_b200 import binding as b

    gamma, x = torch.rand(D, device="cuda") + 0.5, mk(T, D + 8)[:, :D]
    want, saved = b.nvfp4_layernorm_fwd(x, gamma, save=save)
    got, kept = b.nvfp4_layernorm_fwd(x, gamma, save=save, out=x)
    assert got is x and torch.equal(x, want)
    if save:
        assert torch.equal(saved.x8.buf, kept.x8.buf) and torch.equal(saved.stats, kept.stats)
