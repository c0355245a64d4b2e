"""The bias gradient of a layer with more outputs than a launch of 16 columns a workgroup holds."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [0, 1])
def test_a_wide_bias_gradient_is_added_to_what_is_there(K):
    """2^28 + 100 columns, 16 for each of 256 threads, are more than 2^32 threads."""
    import paper_2601_01473_amd as ag
    N = (1 << 28) + 100
    g = torch.randint(-64, 65, (2, N), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    kept = ag.mx8_quantize(torch.ones(2, K, device="cuda"))
    out, bias = torch.full((N, K), 3.0, device="cuda"), torch.full((N,), 5.0, device="cuda")
    ag.mx8_weight_grad(g, kept, bias=True, out=out, bias_out=bias, accumulate=True)
    want = g[0].float() + g[1].float()                      # whole numbers
    assert torch.equal(bias, want + 5)
    if K:
        assert torch.equal(out[:, 0], want + 3)
