"""Every tile of the 8-bit product and of the weight gradient from kept rows: sizes that the rules send to it, with
remainders on each side; and gradients whose results are exact, to the bit."""
import pytest
import torch

from tests import more_operators_ref as ref
from tests import tile_rules
from tests.operators_ref import FLOATS, within

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def ag():
    import paper_2601_01473_amd as m
    return m


def rows_of(R, K, dtype=F32, seed=1, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(R, K, generator=g) * torch.exp(spread * torch.randn(R, 1, generator=g))).to(dtype).cuda()


# ----------------------------------------------------------------- 8-bit product

@pytest.mark.parametrize("tile,M,N,K", [(256, 4000, 4001, 600), (256, 3000, 4097, 2070), (128, 2500, 2303, 700),
                                        (128, 5000, 4900, 100), (64, 1000, 1101, 2000), (64, 60, 301, 4000), (0, 13, 500, 900)])
@pytest.mark.parametrize("out", FLOATS)
def test_product_tiles(ag, tile, M, N, K, out):
    assert tile_rules.int8(M, N, K)[0] == tile
    x, w, b = rows_of(M, K, BF16, spread=2.0), rows_of(N, K, seed=2) / K ** 0.5, torch.randn(N, device="cuda")
    q = ag.int8_quantize(w)
    y, err = ref.int8_product(*ref.int8(x), q.codes, q.scales, K, b, True)
    wide = torch.full((M + 2, N + 5), 3.0, dtype=out, device="cuda")
    got = ag.int8_linear(x, q, b, relu=True, out=wide[1:M + 1, 2:2 + N])
    within(got, y, err, "%d x %d x %d" % (M, N, K))
    assert torch.equal(ag.int8_linear(ag.int8_quantize(x), q, b, relu=True, dtype=out), got)
    wide[1:M + 1, 2:2 + N] = 3.0
    assert bool((wide == 3).all())


# ----------------------------------------------------------------- weight gradient

# way, rows and columns of a tile, whether the rows are cut in parts; M, N, K, the gradient's type
TILES = [("direct", 256, 256, False, 300, 4088, 4001, BF16), ("cut", 256, 256, False, 270, 4087, 4000, BF16),
         ("cut", 128, 256, False, 300, 3001, 3000, F16), ("cut", 128, 256, False, 300, 3000, 3001, F32),
         ("cut", 128, 256, True, 2000, 1500, 1501, F16), ("cut", 128, 128, True, 9000, 250, 521, F32),
         ("direct", 128, 128, True, 4000, 1000, 2001, BF16), ("direct", 128, 128, False, 330, 2600, 2201, BF16),
         ("direct", 64, 64, True, 6000, 520, 265, BF16), ("cut", 64, 64, True, 9000, 250, 521, F16),
         ("cut", 64, 64, True, 2300, 1001, 261, F32), ("registers", 64, 64, False, 200, 130, 101, F32),
         ("registers", 64, 64, False, 200, 131, 100, F16), ("registers", 64, 64, False, 200, 129, 70, BF16)]


def takes(g, K, way, rows, cols, parts):
    got = tile_rules.weight_grad(g, K)
    assert got[:3] == (way, rows, cols) and (got[3] > 1) == parts, got


@pytest.mark.parametrize("way,rows,cols,parts,M,N,K,dtype", TILES)
@pytest.mark.parametrize("out", [F32, BF16])
def test_weight_gradient_tiles(ag, way, rows, cols, parts, M, N, K, dtype, out):
    g, x = rows_of(M, N, dtype), rows_of(M, K, seed=2)
    takes(g, K, way, rows, cols, parts)
    kept = ag.mx8_quantize(x)
    old, old_b = rows_of(N, K, out, seed=3), torch.randn(N, device="cuda")
    values = ref.mx8_values(kept.codes, kept.scales, K)
    W, eW, b, eb = ref.weight_grad(g, values)
    wide = torch.full((N + 2, K + 5), 3.0, dtype=out, device="cuda")
    got, db = ag.mx8_weight_grad(g, kept, bias=True, out=wide[1:N + 1, 2:2 + K])
    within(got, W, eW, "weight gradient")
    within(db, b, eb, "bias gradient")
    W, eW, b, eb = ref.weight_grad(g, values, old, old_b)
    got.copy_(old)
    ag.mx8_weight_grad(g, kept, bias=True, out=got, bias_out=old_b, accumulate=True)
    within(got, W, eW, "added to the weight gradient")
    within(old_b, b, eb, "added to the bias gradient")
    got.fill_(3.0)
    assert bool((wide == 3).all())


@pytest.mark.parametrize("way,rows,cols,parts,M,N,K,dtype", TILES)
def test_exact_weight_gradients(ag, way, rows, cols, parts, M, N, K, dtype):
    """One gradient per column, with all the digits of its type, and kept values that are powers of two: every result
    is one product, and the sum of its pieces is exact in any order."""
    gen = torch.Generator().manual_seed(7)
    at = torch.randint(M, (N,), generator=gen)
    value = (1 + torch.rand(N, generator=gen)) * torch.exp2(torch.randint(-8, 8, (N,), generator=gen).float())
    value = (value * (1 - 2 * torch.randint(2, (N,), generator=gen))).to(dtype)
    g = torch.zeros(M, N, dtype=dtype)
    g[at, torch.arange(N)] = value
    g = g.cuda()
    takes(g, K, way, rows, cols, parts)
    # down to 1/64 of the block's scale: codes 1 .. 64
    x = torch.exp2(torch.randint(-6, 1, (M, K), generator=gen).float()) * (1 - 2 * torch.randint(2, (M, K), generator=gen))
    x[:, ::32] = 1.0
    x *= torch.exp2(torch.randint(-20, 20, (M, 1), generator=gen).float())
    kept = ag.mx8_quantize(x.cuda())
    got, db = ag.mx8_weight_grad(g, kept, bias=True, dtype=F32)
    assert torch.equal(got.cpu(), value.float().unsqueeze(1) * x[at])
    assert torch.equal(db.cpu(), value.float())
