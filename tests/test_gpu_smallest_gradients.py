"""The weight gradient from gradients next to the smallest numbers of their types, to the bit."""
import pytest
import torch

from tests import tile_rules

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def ag():
    import paper_2601_01473_amd as m
    return m


@pytest.mark.parametrize("M,N,K,way", [(200, 130, 100, "registers"), (9000, 250, 521, "cut"), (300, 3000, 3001, "cut")])
def test_smallest_gradients(ag, M, N, K, way):
    """A float32 gradient's digits count down to 2^-133, the smallest bfloat16: from 2^-110 on up that is all of them,
    below it what lies under 2^-133 is left out."""
    gen = torch.Generator().manual_seed(8)
    at = torch.randint(M, (N,), generator=gen)
    value = (1 + torch.rand(N, generator=gen)).double() * torch.exp2(-149 + 49 * torch.arange(N).double() / N).log2().floor().exp2()
    value = value.float()                                   # below 2^-126 with fewer digits
    g = torch.zeros(M, N)
    g[at, torch.arange(N)] = value
    assert tile_rules.weight_grad(g, K)[0] == way
    kept = ag.mx8_quantize(torch.full((M, K), 2.0 ** 60, device="cuda"))
    got = ag.mx8_weight_grad(g.cuda(), kept, dtype=F32).cpu()
    counted = torch.floor(value.double() * 2.0 ** 133) * 2.0 ** -133
    assert bool((counted == value)[value >= 2.0 ** -110].all())
    assert torch.equal(got, (counted * 2.0 ** 60).float().unsqueeze(1).expand(N, K))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_smallest_gradients_of_16_bits(ag, dtype):
    """All their numbers have all their digits."""
    bits = torch.arange(1, 1 << 10 if dtype == F16 else 1 << 8, dtype=torch.int16)
    for M in (40, 300):
        N, K = len(bits), 1030
        g = torch.zeros(M, N, dtype=dtype)
        g[torch.arange(N) % M, torch.arange(N)] = bits.view(dtype)
        for shift in (0, 1):                                # rows of whole pieces, and not
            wide = torch.zeros(M, N + 1, dtype=dtype, device="cuda")
            wide[:, shift:shift + N] = g.cuda()
            kept = ag.mx8_quantize(torch.full((M, K), 2.0 ** 60, device="cuda"))
            got = ag.mx8_weight_grad(wide[:, shift:shift + N], kept, dtype=F32).cpu()
            assert torch.equal(got, (bits.view(dtype).double() * 2.0 ** 60).float().unsqueeze(1).expand(N, K))
