"""Which 8-bit products are refused for their size: by the number of tiles that a launch holds, not by which tile the cost
model prefers.  Workspace sizes are asked for on the host; nothing is launched."""
import pytest

from paper_2601_01473_amd import _binding as B

MOST = (1 << 23) - 8


def refused(M, N, K):
    with pytest.raises(B.AgnesError) as e:
        B.agnes_int8_product_bytes(M, N, K)
    assert e.value.status == B.AGNES_ERR_RANGE, e.value
    with pytest.raises(B.AgnesError) as e:
        B.agnes_int8_linear_bytes(M, N, K)
    assert e.value.status == B.AGNES_ERR_RANGE, e.value


@pytest.mark.parametrize("K", [0, 1, 32, 100, 4096, (1 << 17) - 1])
def test_the_largest_products(K):
    for M in (17, 32, 33, 40, 64, 65, 200, 256):
        for N in ((1 << 27) + 5, 1 << 29, MOST * 256):
            assert B.agnes_int8_product_bytes(M, N, K) == 0
            assert B.agnes_int8_linear_bytes(M, N, K) >= M * K
        refused(M, MOST * 256 + 1, K)
    for M, rows in ((257, 2), (512, 2), (1000, 4), (1 << 20, 1 << 12), (1 << 30, 1 << 22)):
        B.agnes_int8_product_bytes(M, MOST // rows * 256, K)
        refused(M, MOST // rows * 256 + 1, K)
    for M in (1, 16):
        B.agnes_int8_product_bytes(M, MOST * 16, K)
        refused(M, MOST * 16 + 1, K)


@pytest.mark.gpu
def test_a_product_whose_preferred_tiles_are_too_many():
    """Tiles of 64 would be 2^23 + 5."""
    import torch

    import paper_2601_01473_amd as ag
    M, N = 33, (1 << 29) + 300
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(M, 1, device="cuda", generator=g)
    w = ag.int8_quantize(torch.randn(N, 1, device="cuda", generator=g).to(torch.bfloat16))
    got = ag.int8_linear(x, w, dtype=torch.bfloat16)
    q = ag.int8_quantize(x)
    for at in (0, 12345678, 1 << 28, (1 << 29) - 500, N - 1000):
        n = slice(at, at + 1000)
        sums = q.codes[:, :1].float() * w.codes[n, 0].float()       # one product of codes
        assert torch.equal(got[:, n], (sums * q.scales.unsqueeze(1) * w.scales[n]).to(torch.bfloat16))
