"""nvfp4_gemv's waits: bounded, and reported."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def operand(N, K):
    from paper_2510_27527_b200 import binding as b

    return b.nvfp4_quantize((torch.randn(N, K, device="cuda") * 0.02).bfloat16())


@pytest.mark.parametrize("M", [1, 2, 3, 4, 7, 16, 32])
@pytest.mark.parametrize("N,K", [(100, 256), (300, 4096)])  # one CTA to a row tile; clusters
def test_a_wait_that_runs_out_ends_the_kernel_with_a_status(M, N, K):
    """The first stage is made to expect bytes that never arrive and the bound is about a millisecond: the kernel returns and reports it, and the
    same product right afterwards is correct."""
    from paper_2510_27527_b200 import binding as b

    W, x = operand(N, K), torch.randn(M, K, device="cuda").bfloat16()
    want = b.nvfp4_gemv(x, W, b.DT_F32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    b.nvfp4_gemv_ex(x, W, b.DT_F32, status, wait_limit_cycles=2_000_000, starve_first_stage=True)
    torch.cuda.synchronize()
    assert int(status) == b.ERR_TIMEOUT
    status.zero_()
    assert torch.equal(b.nvfp4_gemv_ex(x, W, b.DT_F32, status, wait_limit_cycles=200_000_000), want) and int(status) == 0
    assert torch.equal(b.nvfp4_gemv(x, W, b.DT_F32, dev_status=status), want) and int(status) == 0


def test_a_frozen_layer_keeps_its_layers_status_word(monkeypatch):
    from paper_2510_27527_b200 import binding as b
    from paper_2510_27527_b200.block import NVFP4MLP
    from paper_2510_27527_b200.module import NVFP4Linear

    words = []

    class Seen:
        def __getattr__(self, name):
            return getattr(node, name)

        def gemv(self, *args):
            words.append(args[14])
            return node.gemv(*args)

    node, status = b._node, torch.zeros(1, dtype=torch.int32, device="cuda")
    monkeypatch.setattr(b, "_node", Seen())
    x = torch.randn(2, 64, device="cuda").bfloat16()
    with torch.no_grad():
        NVFP4Linear(64, 32, cfg=b.LayerConfig(dev_status=status)).frozen()(x)
        NVFP4MLP(64, 128, b.LayerConfig(dev_status=status)).frozen()(x)
        assert len(words) == 4 and all(w is status for w in words)
        NVFP4Linear(64, 32).frozen()(x)
        assert words[-1] is None


def test_status_words_of_another_kind_are_refused():
    from paper_2510_27527_b200 import binding as b

    W, x = operand(32, 64), torch.randn(2, 64, device="cuda").bfloat16()
    for word in (torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32), torch.zeros(0, dtype=torch.int32, device="cuda")):
        with pytest.raises(RuntimeError, match="dev_status"):
            b.nvfp4_gemv(x, W, dev_status=word)
