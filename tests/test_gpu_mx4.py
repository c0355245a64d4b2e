"""4-bit rows and products on the GPU against the definition in 64 bits (tests/operators_ref.py)."""
import pytest
import torch

from tests import operators_ref as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ag():
    import paper_2601_01473_amd as m
    return m


def normal(shape, dtype, seed, spread=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g)
    if spread:
        x = x * torch.exp(spread * torch.randn(*shape, generator=g))
    return x.to(dtype).cuda()


# ----------------------------------------------------------------- quantisation

def check_quantize(ag, x):
    q = ag.mx4_quantize(x)
    codes, scales = ref.mx4(x)
    assert torch.equal(q.scales.cpu(), scales)
    assert torch.equal(q.codes.cpu(), codes)
    v = ref.mx4_values(codes, scales, x.shape[1])
    for dtype in ref.FLOATS:
        ref.within(ag.mx4_dequantize(q, dtype=dtype), v, torch.zeros_like(v), "values")
    return q


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (1, 32), (3, 33), (5, 64), (2, 129), (7, 250), (1, 1003), (40, 96),
                                       (3, 2048)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_quantize(ag, rows, cols, dtype):
    check_quantize(ag, normal((rows, cols), dtype, 1, spread=1.0))


def test_quantize_ties_signs_and_zeros(ag):
    """Every midpoint, both signs, and the values next to it, under several scales."""
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 4.0, 0.0, 0.5]
    rows = []
    for e in (-100, -20, 0, 1, 30, 120):
        for m in mids:
            v = torch.tensor([m], dtype=F32)
            near = [float(v), float(torch.nextafter(v, torch.tensor(INF))), float(torch.nextafter(v, torch.tensor(-INF)))]
            block = [s * x * 2.0 ** e for x in near for s in (1, -1)] + [4.0 * 2.0 ** e, -0.0]
            rows.append(block + [0.0] * (32 - len(block)))
    check_quantize(ag, torch.tensor(rows, dtype=F32, device="cuda"))


def test_quantize_extremes(ag):
    tiny, big = 2.0 ** -149, torch.finfo(F32).max
    rows = [[0.0] * 32, [tiny] * 32, [-tiny] + [0.0] * 31, [2.0 ** -126] * 32, [2.0 ** -125, 2.0 ** -127, 2.0 ** -128] + [0.0] * 29,
            [big, -big] + [1.0] * 30, [2.0 ** 127] * 32, [6.0 * 2.0 ** -127, 2.0 ** -128] + [0.0] * 30, [-0.0] * 32]
    check_quantize(ag, torch.tensor(rows, dtype=F32, device="cuda"))
    low = torch.finfo(F16)
    check_quantize(ag, torch.tensor([[low.max, low.min, low.tiny, 2.0 ** -24] * 8], dtype=F16, device="cuda"))


def test_quantize_nan_and_infinity_mark_their_block(ag):
    x = normal((4, 100), F32, 2)
    x[0, 3], x[1, 40], x[2, 99] = NAN, INF, -INF
    q = check_quantize(ag, x)
    v = ag.mx4_dequantize(q)
    nan = v.isnan()
    assert bool(nan[0, :32].all()) and bool(nan[1, 32:64].all()) and bool(nan[2, 96:].all()) and int(nan.sum()) == 68


def test_quantize_strides(ag):
    wide = normal((20, 200), BF16, 3)
    for view in (wide[:, 5:105], wide[::2, 1:34], wide[:1, :90].expand(6, 90)):
        check_quantize(ag, view)
    q = ag.mx4_quantize(wide)
    assert ag.mx4_dequantize(q, dtype=F16).shape == (20, 200)


def test_quantize_empty(ag):
    for shape in ((0, 40), (3, 0)):
        q = ag.mx4_quantize(torch.empty(*shape, device="cuda"))
        assert ag.mx4_dequantize(q).shape == shape


def test_quantize_again_changes_nothing(ag):
    """Values that are exact in the format keep their value, if a block's largest has the exponent that set its scale."""
    x = normal((50, 320), F32, 4, spread=2.0)
    once = ag.mx4_dequantize(ag.mx4_quantize(x))
    assert torch.equal(ag.mx4_dequantize(ag.mx4_quantize(once)), once)


# ----------------------------------------------------------------- product

def check_linear(ag, M, N, K, dtype=BF16, out=None, bias=True, relu=False, seed=5):
    x, w = normal((M, K), dtype, seed, spread=0.5), normal((N, K), F32, seed + 1)
    b = normal((N,), F32, seed + 2) if bias else None
    qx, qw = ag.mx4_quantize(x), ag.mx4_quantize(w)
    vx, vw = (ref.mx4_values(q.codes, q.scales, K) for q in (qx, qw))
    want, err = ref.product(vx, vw, b, relu)
    got = ag.mx4_linear(x, qw, b, relu=relu, dtype=out)
    assert got.dtype == (out or dtype)
    ref.within(got, want, err, "linear %d %d %d" % (M, N, K))
    ref.within(ag.mx4_linear(qx, qw, b, relu=relu), want, err, "product")
    return got


@pytest.mark.parametrize("M", [1, 2, 5, 16, 17, 33, 100, 130, 257])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 32), (17, 33), (64, 128), (130, 250), (96, 1024), (300, 2080)])
def test_linear_sizes(ag, M, N, K):
    check_linear(ag, M, N, K)


@pytest.mark.parametrize("M,N,K", [(512, 768, 512), (257, 1031, 640), (1, 4096, 4096), (3, 5000, 3000), (1025, 513, 96),
                                   (16, 128, 8192), (40, 2048, 8192), (700, 8, 4096), (2000, 260, 4128)])
def test_linear_larger(ag, M, N, K):
    check_linear(ag, M, N, K)
    check_linear(ag, M, N, K, dtype=F32, bias=False)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("out", [F32, F16, BF16])
@pytest.mark.parametrize("M", [2, 70])
def test_linear_every_pair_of_types(ag, dtype, out, M):
    check_linear(ag, M, 90, 200, dtype=dtype, out=out, relu=True)
    check_linear(ag, M, 90, 200, dtype=dtype, out=out, bias=False)


def test_linear_whole_numbers_are_exact(ag):
    """Operands of the format's own values and sums below 2^24: no rounding anywhere."""
    g = torch.Generator().manual_seed(6)
    grid = torch.tensor(ref.MAGNITUDES + [-m for m in ref.MAGNITUDES])
    for M, N, K in ((1, 50, 4096), (9, 64, 4096), (130, 140, 4096), (300, 300, 1056)):
        x, w = grid[torch.randint(0, 16, (M, K), generator=g)], grid[torch.randint(0, 16, (N, K), generator=g)]
        x[:, ::32], w[:, ::32] = 6, 4                        # every block's scale is 1
        got = ag.mx4_linear(x.cuda(), ag.mx4_quantize(w.cuda()))
        assert torch.equal(got.cpu().double(), x.double() @ w.double().T)


def test_linear_every_scale_reaches_its_block(ag):
    """One nonzero block per row, with a scale of its own: each product is a single block's."""
    K = 32 * 70
    x, w = torch.zeros(140, K), torch.ones(64, K)
    for r in range(140):
        b = r % 70
        x[r, 32 * b:32 * b + 32] = 2.0 ** (r - 70)
    for n in range(64):
        w[n] *= 2.0 ** (n % 9 - 4)
    for rows in (x, x[:3], x[69:74], x[100:117]):
        got = ag.mx4_linear(rows.cuda(), ag.mx4_quantize(w.cuda()))
        assert torch.equal(got.cpu().double(), rows.double() @ w.double().T)


@pytest.mark.parametrize("M", [1, 4, 40, 300])
def test_linear_nan_blocks(ag, M):
    """A block with an infinity or NaN makes its whole row (of x) or column (of w) NaN, and nothing else; also after relu."""
    x, w = normal((M, 300), F32, 7), normal((70, 300), F32, 8)
    x[M - 1, 290], w[5, 3], w[64, 150] = INF, NAN, -INF
    for relu in (False, True):
        got = ag.mx4_linear(x, ag.mx4_quantize(w), relu=relu).cpu()
        nan = torch.zeros(M, 70, dtype=torch.bool)
        nan[M - 1], nan[:, 5], nan[:, 64] = True, True, True
        assert torch.equal(got.isnan(), nan)


def test_linear_without_columns(ag):
    b = normal((5,), F32, 9)
    w = ag.mx4_quantize(torch.empty(5, 0, device="cuda"))
    assert torch.equal(ag.mx4_linear(torch.empty(3, 0, device="cuda"), w, b), b.expand(3, 5))
    assert ag.mx4_linear(torch.empty(0, 64, device="cuda"), ag.mx4_quantize(normal((5, 64), F32, 1))).shape == (0, 5)
    assert ag.mx4_linear(torch.empty(3, 64, device="cuda"), ag.mx4_quantize(torch.empty(0, 64, device="cuda"))).shape == (3, 0)


@pytest.mark.parametrize("M", [1, 7, 200])
def test_linear_strides(ag, M):
    wide = normal((M, 500), BF16, 10)
    x, w, b = wide[:, 3:203], normal((90, 200), F32, 11), normal((90,), F32, 12)
    q = ag.mx4_quantize(w)
    out = torch.full((M, 133), 5.0, dtype=F16, device="cuda")
    ag.mx4_linear(x, q, b, out=out[:, 7:97])
    assert torch.equal(out[:, 7:97], ag.mx4_linear(x.contiguous(), q, b, dtype=F16))
    assert bool((out[:, :7] == 5).all()) and bool((out[:, 97:] == 5).all())


def test_linear_offsets_past_32_bits(ag):
    """More than 2^31 outputs; x's codes are all the same, so every row equals the first."""
    M, N = 70000, 32000
    x = normal((1, 64), BF16, 13).expand(M, 64)
    w = ag.mx4_quantize(normal((N, 64), F32, 14))
    out = ag.mx4_linear(x, w)
    want, err = ref.product(ref.mx4_values(*ag.mx4_quantize(x[:1])), ref.mx4_values(*w), None, False)
    for r in (0, 1, 67107, 67108, 67109, M - 1):
        ref.within(out[r:r + 1], want, err)
    for r in range(0, M, 10000):
        assert bool((out[r:r + 10000] == out[0]).all())


def test_linear_same_bits_every_time_and_on_another_stream(ag):
    for M, N, K in ((1, 300, 4096), (8, 4096, 4096), (300, 400, 1000)):
        x, w, b = normal((M, K), BF16, 15), ag.mx4_quantize(normal((N, K), F32, 16)), normal((N,), F32, 17)
        want = ag.mx4_linear(x, w, b)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = [ag.mx4_linear(x, w, b, stream=side) for _ in range(3)]
        side.synchronize()
        assert all(torch.equal(g, want) for g in got)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = ag.mx4_linear(x, w, b)
            back = ag.mx4_dequantize(ag.mx4_quantize(x))
        for k in range(3):
            x.copy_(normal((M, K), BF16, 20 + k))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ag.mx4_linear(x, w, b))
            assert torch.equal(back, ag.mx4_dequantize(ag.mx4_quantize(x)))


@pytest.mark.parametrize("M", [16, 17, 31, 32, 33, 48, 64, 65])
@pytest.mark.parametrize("N,K", [(70, 300), (100, 4096), (33, 4129), (4100, 2048)])
def test_linear_rows_about_the_limits_of_the_kernels(ag, M, N, K):
    """The kernel of few rows, whole tiles and parts of K take over from each other about here."""
    check_linear(ag, M, N, K, bias=M % 2 == 0, relu=M == 33)


def test_quantize_more_than_one_launch_holds(ag):
    """One row of 8192 for 2^24 + 5 rows: a workgroup each, more than a launch takes; 69 GB of codes."""
    rows, K = (1 << 24) + 5, 8192
    torch.cuda.empty_cache()
    one = normal((1, K), BF16, 22, spread=1.0)
    codes, scales = ref.mx4(one)
    q = ag.mx4_quantize(one.expand(rows, K))
    for r in range(0, rows, 1 << 20):
        assert bool((q.codes[r:r + (1 << 20)] == codes.cuda()).all()), r
        assert bool((q.scales[r:r + (1 << 20)] == scales.cuda()).all()), r
    del q
    torch.cuda.empty_cache()


def test_rows_on_both_sides_of_a_launch(ag):
    """Narrow rows, 2^30 of them in a launch: back and forth across the boundary."""
    rows, at = (1 << 30) + 3, (1 << 30) - 2
    torch.cuda.empty_cache()
    x = torch.zeros(rows, 1, dtype=BF16, device="cuda")
    x[:3, 0], x[at:, 0] = torch.tensor([1.5, -3.0, 0.25]).to(BF16).cuda(), torch.tensor([0.5, -6.0, 4.0, -1.0, 3.0]).to(BF16).cuda()
    v = ag.mx4_dequantize(ag.mx4_quantize(x), dtype=BF16)
    assert torch.equal(v[:3], x[:3]) and torch.equal(v[at:], x[at:])      # of the format's values, each its block's largest
    assert int((v != 0).sum()) == 8
    del x, v
    torch.cuda.empty_cache()


def test_linear_of_more_than_2_to_26_columns(ag):
    """The header's limit is 2^23 tiles; of one row a tile is 16 columns wide."""
    N, K = (1 << 26) + 37, 32
    g = torch.Generator(device="cuda").manual_seed(23)
    codes = torch.randint(0, 256, (N, 16), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.full((N, 1), 127, dtype=torch.uint8, device="cuda")
    x = normal((2, K), BF16, 24)
    vx = ref.mx4_values(*ag.mx4_quantize(x))
    for rows in (x[:1], ag.mx4_quantize(x)):
        out = ag.mx4_linear(rows, ag.Mx4(codes, scales, K), dtype=F32)
        at = torch.tensor([0, 1, 15, 16, (1 << 25) - 1, (1 << 26) - 1, 1 << 26, N - 17, N - 1], device="cuda")
        want, err = ref.product(vx[:out.shape[0]], ref.mx4_values(codes[at], scales[at], K), None, False)
        ref.within(out[:, at], want, err, "many columns")


# 128 x 128 tiles serve products with at least 256 of them and fewer than 256 of 256 x 256, which serve the rest.  A
# step is 256 columns: none, one, even and odd numbers of them, with and without a part of one behind.
TILES_128 = [(2100, 2100, 1100), (2049, 2047, 1280), (2048, 2048, 512), (1300, 3500, 700), (2100, 2100, 200),
             (2049, 2100, 256)]
TILES_256 = [(4100, 4100, 300), (4100, 4100, 800), (4097, 4095, 1056), (4096, 4096, 2048), (4097, 4200, 250),
             (8200, 2050, 512), (4351, 4097, 256), (4100, 4100, 1792)]


@pytest.mark.parametrize("M,N,K", TILES_128 + TILES_256)
def test_linear_large_tiles(ag, M, N, K):
    check_linear(ag, M, N, K)
    check_linear(ag, M, N, K, dtype=F16, out=F32, bias=False, relu=True, seed=31)


@pytest.mark.parametrize("M,N,K", [TILES_128[0], TILES_128[1], TILES_256[1], TILES_256[2], TILES_256[7]])
def test_linear_large_tiles_whole_numbers_are_exact(ag, M, N, K):
    g = torch.Generator().manual_seed(25)
    grid = torch.tensor(ref.MAGNITUDES + [-m for m in ref.MAGNITUDES])
    x, w = grid[torch.randint(0, 16, (M, K), generator=g)], grid[torch.randint(0, 16, (N, K), generator=g)]
    x[:, ::32], w[:, ::32] = 6, 4                            # every block's scale is 1
    got = ag.mx4_linear(x.cuda(), ag.mx4_quantize(w.cuda()))
    assert torch.equal(got.cpu().double(), x.double() @ w.double().T)
    # rows at other strides, 16-bit results
    out = torch.full((M, N + 9), 5.0, dtype=F16, device="cuda")
    ag.mx4_linear(x.cuda(), ag.mx4_quantize(w.cuda()), out=out[:, 3:3 + N])
    assert torch.equal(out[:, 3:3 + N], got.half())
    assert bool((out[:, :3] == 5).all()) and bool((out[:, 3 + N:] == 5).all())


@pytest.mark.parametrize("M,N", [(2100, 2100), (4100, 4100)])
@pytest.mark.parametrize("blocks", [70, 33])
def test_linear_large_tiles_every_scale_reaches_its_block(ag, M, N, blocks):
    """One nonzero block per row, with a scale of its own, and columns of other scales."""
    K = 32 * blocks
    r, n = torch.arange(M), torch.arange(N)
    x, w = torch.zeros(M, blocks, 32), torch.ones(N, blocks, 32)
    size = 2.0 ** (r * 7 % 101 - 50).double()
    x[r, r % blocks] = size.float().unsqueeze(1)
    power = (n.unsqueeze(1) * 3 + torch.arange(blocks) * 5) % 19 - 9
    w *= (2.0 ** power.double()).float().unsqueeze(2)
    got = ag.mx4_linear(x.view(M, K).cuda(), ag.mx4_quantize(w.view(N, K).cuda()))
    want = 32 * size.unsqueeze(1) * (2.0 ** power.double()).T[r % blocks]
    assert torch.equal(got.cpu().double(), want)
