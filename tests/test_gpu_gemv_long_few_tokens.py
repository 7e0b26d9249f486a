"""Three and four tokens over a long k take the form with X staged in memory, whatever the number of rows: their order of sums is then that of five."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,K,staged", [(128, 30000, True), (512, 14336, True), (1024, 8192, True), (128, 2048, False), (1024, 4096, False)])
def test_the_form_follows_the_pairs_of_a_cta(N, K, staged):
    from paper_2510_27527_b200 import binding as b

    W, x = b.nvfp4_quantize((torch.randn(N, K, device="cuda") * 0.02).bfloat16()), torch.randn(5, K, device="cuda").bfloat16()
    before = b.lib.nvfp4_launch_count()
    y = b.nvfp4_gemv(x[:4], W, b.DT_F32)
    assert b.lib.nvfp4_launch_count() - before == (2 if staged else 1)
    if staged:
        assert torch.equal(y, b.nvfp4_gemv(x, W, b.DT_F32)[:4])
