"""8-bit checkpoints on the GPU, and their use in the backward pass, against definitions in 64 bits
(tests/more_operators_ref.py)."""
import pytest
import torch

from tests import more_operators_ref as ref
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


def same(q, codes, scales):
    assert torch.equal(q.codes.cpu(), codes)
    assert torch.equal(q.scales.cpu(), scales)


@pytest.mark.parametrize("R,K", [(1, 1), (3, 31), (2, 32), (5, 33), (70, 63), (4, 1003), (2, 4096), (1000, 40), (300, 2050)])
@pytest.mark.parametrize("dtype", FLOATS)
def test_kept_rows_and_back(ag, R, K, dtype):
    x = rows_of(R, K, dtype, spread=2.0)
    codes, scales = ref.mx8(x)
    q = ag.mx8_quantize(x)
    same(q, codes, scales)
    values = ref.mx8_values(codes, scales, K)
    for t in FLOATS:
        within(ag.mx8_dequantize(q, t), values, 0.0 * values, "values")
    assert torch.equal(ag.mx8_dequantize(q, BF16).cpu().double(), values)      # exact in bfloat16


def test_extreme_blocks(ag):
    x = torch.zeros(14, 40)
    tiny = 2.0 ** -149
    x[1, 3] = tiny
    x[2] = tiny * torch.arange(40)
    x[3] = 2.0 ** -127 * torch.linspace(-1, 1, 40)
    x[4] = 2.0 ** -126 * torch.linspace(-1.9, 1.9, 40)
    x[5] = torch.finfo(F32).max * torch.linspace(-1, 1, 40)
    x[6] = torch.finfo(F32).min
    x[7, 7], x[8, 39], x[9, 0] = float("nan"), float("inf"), float("-inf")
    x[10] = -0.0
    x[11, 0], x[11, 1], x[11, 2], x[11, 3] = 1.0, 0.5 / 64, 1.5 / 64, -2.5 / 64     # ties to the even code
    x[12, 0], x[12, 1] = 127.5 / 64, -127.75 / 64           # above 127
    x[13, :32] = 1.0
    x[13, 32:] = 2.0 ** -60
    codes, scales = ref.mx8(x)
    q = ag.mx8_quantize(x.cuda())
    same(q, codes, scales)
    values = ref.mx8_values(codes, scales, 40)
    within(ag.mx8_dequantize(q), values, 0.0 * values)
    assert ag.mx8_quantize(x[:0].cuda()).codes.shape == (0, 64)
    assert ag.mx8_dequantize(ag.mx8_quantize(torch.zeros(3, 0, device="cuda"))).shape == (3, 0)


# ----------------------------------------------------------------- activations

def check_act(ag, x, g, act, gated, ty=None, tx=None, what=""):
    y, kept = ag.mx8_activation(x, act, gated=gated, dtype=ty)
    Y, eY = ref.activation(act, x, gated)
    within(y, Y, eY, what + " y")
    codes, scales = ref.mx8(x)
    same(kept, codes, scales)
    alone, none = ag.mx8_activation(x, act, gated=gated, keep=False, dtype=ty)
    assert none is None and torch.equal(alone, y)
    dx = ag.mx8_activation_grad(g, kept, act, gated=gated, dtype=tx)
    D, eD = ref.activation_grad(act, g, ref.mx8_values(codes, scales, x.shape[1]), gated)
    within(dx, D, eD, what + " dx")
    return y, dx


@pytest.mark.parametrize("R,F", [(1, 1), (1, 32), (3, 31), (2, 33), (5, 40), (70, 64), (4, 1003), (3, 1024), (600, 256),
                                 (2, 8192), (1000, 8)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", FLOATS)
def test_activations(ag, R, F, act, gated, dtype):
    x, g = rows_of(R, F * (2 if gated else 1), dtype, spread=1.0), rows_of(R, F, dtype, seed=2)
    check_act(ag, x, g, act, gated)


@pytest.mark.parametrize("tx", FLOATS)
@pytest.mark.parametrize("ty", FLOATS)
@pytest.mark.parametrize("gated", [False, True])
def test_every_pair_of_types(ag, tx, ty, gated):
    for F in (64, 45):
        x = rows_of(7, F * (2 if gated else 1), tx)
        for tg in FLOATS:
            check_act(ag, x, rows_of(7, F, tg, seed=2), "silu", gated, ty=ty, tx=ty)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_whole_range_of_the_argument(ag, act):
    x = torch.cat([torch.linspace(-200, 200, 4001), torch.linspace(-6, 6, 4001),
                   torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3e38, -3e38, 2.0 ** -149])])
    x = torch.nn.functional.pad(x, (0, -len(x) % 32)).view(-1, 1).cuda()           # one element per block
    check_act(ag, x, torch.ones_like(x), act, False)
    both = torch.cat([x, torch.full_like(x, 3.0)], 1)
    check_act(ag, both, torch.ones_like(x), act, True)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("F", [64, 50])
def test_undefined_blocks(ag, gated, F):
    """A NaN spoils its own value going forward and its block going back, and nothing else."""
    x, g = rows_of(4, F * (2 if gated else 1)), rows_of(4, F, seed=2)
    x[1, 3] = float("nan")
    y, kept = ag.mx8_activation(x, "silu", gated=gated)
    bad = torch.zeros(4, F, dtype=torch.bool)
    bad[1, 3] = True
    assert torch.equal(torch.isnan(y.cpu()), bad)
    dx = ag.mx8_activation_grad(g, kept, "silu", gated=gated)
    bad = torch.zeros(4, F * (2 if gated else 1), dtype=torch.bool)
    bad[1, :32] = True
    if gated:
        bad[1, F:F + 32] = True
    assert torch.equal(torch.isnan(dx.cpu()), bad)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("F", [64, 51])
def test_strides_and_untouched_memory(ag, gated, F):
    cols = F * (2 if gated else 1)
    wide, gw = torch.randn(9, cols + 9, device="cuda"), torch.randn(9, F + 5, device="cuda", dtype=BF16)
    x, g = wide[:, 4:4 + cols], gw[:, 1:1 + F]
    y, kept = ag.mx8_activation(x.contiguous(), "gelu", gated=gated)
    dx = ag.mx8_activation_grad(g.contiguous(), kept, "gelu", gated=gated)
    out, dout = torch.full((9, F + 3), 3.0, device="cuda"), torch.full((9, cols + 3), 3.0, device="cuda", dtype=BF16)
    y2, kept2 = ag.mx8_activation(x, "gelu", gated=gated, out=out[:, 1:1 + F])
    ag.mx8_activation_grad(g, kept2, "gelu", gated=gated, out=dout[:, 2:2 + cols])
    assert torch.equal(out[:, 1:1 + F], y) and torch.equal(dout[:, 2:2 + cols], dx)
    assert torch.equal(kept.codes, kept2.codes) and torch.equal(kept.scales, kept2.scales)
    out[:, 1:1 + F] = 3
    dout[:, 2:2 + cols] = 3
    assert bool((out == 3).all()) and bool((dout == 3).all())
    # the gradient of a sum is an expanded scalar
    one = torch.ones(1, 1, device="cuda").expand(9, F)
    within(ag.mx8_activation_grad(one, kept, "gelu", gated=gated),
           *ref.activation_grad("gelu", one, ref.mx8_values(*kept[:2], cols), gated))
    assert ag.mx8_activation(x[:0], "gelu", gated=gated)[0].shape == (0, F)


def test_activation_gradient_against_differences(ag):
    """The slope at the kept values, against central differences of the definition."""
    for act in ("silu", "gelu"):
        x = rows_of(6, 64)
        _, kept = ag.mx8_activation(x, act, gated=True)
        g = rows_of(6, 32, seed=4)
        dx = ag.mx8_activation_grad(g, kept, act, gated=True).cpu().double()
        k, h = ref.mx8_values(*kept[:2], 64), 1e-5
        for j in (0, 5, 31, 32, 50, 63):
            up, down = k.clone(), k.clone()
            up[:, j] += h
            down[:, j] -= h
            num = ((ref.activation(act, up, True)[0] - ref.activation(act, down, True)[0]) * g.cpu().double()).sum(1) / (2 * h)
            # h^2 / 6 of the third derivative and 1e-16 / h of rounding, on values below 1000
            assert float((dx[:, j] - num).abs().max()) < 1e-6 * max(1.0, float(k.abs().max() * g.abs().max()))


# ----------------------------------------------------------------- weight gradient

def check_wgrad(ag, M, N, K, dtype, out, seed=1, bias=True):
    g, x = rows_of(M, N, dtype, seed), rows_of(M, K, F32, seed + 1)
    kept = ag.mx8_quantize(x)
    W, eW, b, eb = ref.weight_grad(g, ref.mx8_values(kept.codes, kept.scales, K))
    got = ag.mx8_weight_grad(g, kept, bias=bias, dtype=out)
    if bias:
        got, db = got
        assert db.dtype == F32
        within(db, b, eb, "bias gradient %d %d %d" % (M, N, K))
    within(got, W, eW, "weight gradient %d %d %d" % (M, N, K))
    return g, kept, got


WSIZES = [(1, 1, 1), (2, 3, 5), (31, 16, 32), (32, 47, 256), (33, 17, 100), (64, 64, 64), (100, 130, 70), (257, 300, 129),
          (500, 256, 256), (1000, 5, 700), (2048, 47, 256), (3001, 65, 33), (130, 600, 515), (70, 1100, 1030),
          (20000, 8, 8), (5000, 200, 300), (96, 2, 3000), (65, 3000, 2), (40, 4200, 4100)]


@pytest.mark.parametrize("M,N,K", WSIZES)
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F32, F32), (F16, F16), (BF16, BF16)])
def test_weight_gradients(ag, M, N, K, dtype, out):
    check_wgrad(ag, M, N, K, dtype, out, bias=N != 64)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("out", FLOATS)
@pytest.mark.parametrize("M,N,K", [(50, 70, 90), (4000, 40, 64)])
def test_accumulated_weight_gradients(ag, dtype, out, M, N, K):
    g, kept, _ = check_wgrad(ag, M, N, K, dtype, out)
    old, old_b = rows_of(N, K, out, seed=5), torch.randn(N, device="cuda")
    W, eW, b, eb = ref.weight_grad(g, ref.mx8_values(kept.codes, kept.scales, K), old, old_b)
    acc, acc_b = old.clone(), old_b.clone()
    got, db = ag.mx8_weight_grad(g, kept, bias=True, out=acc, bias_out=acc_b, accumulate=True)
    assert got is acc and db is acc_b
    within(acc, W, eW)
    within(acc_b, b, eb)


def test_no_rows(ag):
    g, kept = torch.zeros(0, 5, device="cuda"), ag.mx8_quantize(torch.zeros(0, 40, device="cuda"))
    W, b = ag.mx8_weight_grad(g, kept, bias=True)
    assert W.shape == (5, 40) and bool((W == 0).all()) and bool((b == 0).all())
    old, old_b = torch.randn(5, 40, device="cuda"), torch.randn(5, device="cuda")
    acc, acc_b = old.clone(), old_b.clone()
    ag.mx8_weight_grad(g, kept, bias=True, out=acc, bias_out=acc_b, accumulate=True)
    assert torch.equal(acc, old) and torch.equal(acc_b, old_b)
    g = torch.ones(6, 5, device="cuda")
    none = ag.mx8_quantize(torch.zeros(6, 0, device="cuda"))
    W, b = ag.mx8_weight_grad(g, none, bias=True)
    assert W.shape == (5, 0) and bool((b == 6).all())
    W, b = ag.mx8_weight_grad(g[:, :0], ag.mx8_quantize(torch.ones(6, 7, device="cuda")), bias=True)
    assert W.shape == (0, 7) and b.shape == (0,)


@pytest.mark.parametrize("M,N,K", [(40, 50, 70), (700, 300, 290)])
@pytest.mark.parametrize("dtype", FLOATS)
def test_wgrad_strides_and_untouched_memory(ag, M, N, K, dtype):
    wide = rows_of(M, N + 9, dtype)
    g = wide[:, 3:3 + N]
    kept = ag.mx8_quantize(rows_of(M, K))
    want = ag.mx8_weight_grad(g.contiguous(), kept, dtype=F32)
    out = torch.full((N + 2, K + 5), 3.0, device="cuda")
    ag.mx8_weight_grad(g, kept, out=out[1:N + 1, 2:2 + K])
    assert torch.equal(out[1:N + 1, 2:2 + K], want)
    out[1:N + 1, 2:2 + K] = 3.0
    assert bool((out == 3).all())
    # the same gradient for all rows: the gradient of a mean
    one = wide[:1, :N].expand(M, N)
    W, eW, _, _ = ref.weight_grad(one, ref.mx8_values(kept.codes, kept.scales, K))
    within(ag.mx8_weight_grad(one, kept, dtype=F32), W, eW)
    scalar = torch.ones(1, 1, device="cuda", dtype=dtype).expand(M, N)
    W, eW, _, _ = ref.weight_grad(scalar, ref.mx8_values(kept.codes, kept.scales, K))
    within(ag.mx8_weight_grad(scalar, kept, dtype=F32), W, eW)


@pytest.mark.parametrize("dtype", FLOATS)
def test_gradients_of_every_magnitude(ag, dtype):
    """Large, small and infinite gradients: an infinity or NaN stays in its row of the weight's gradient."""
    g = rows_of(300, 40, F32)
    g *= torch.exp2(torch.linspace(-18, 12, 40, device="cuda"))
    if dtype != F16:
        g *= torch.exp2(torch.linspace(-40, 60, 40, device="cuda"))
    g = g.to(dtype)
    kept = ag.mx8_quantize(rows_of(300, 100))
    v = ref.mx8_values(kept.codes, kept.scales, 100)
    W, eW, b, eb = ref.weight_grad(g, v)
    got, db = ag.mx8_weight_grad(g, kept, bias=True, dtype=F32)
    within(got, W, eW)
    within(db, b, eb)
    top = torch.finfo(dtype).max
    g[5, 7], g[6, 8], g[7, 9], g[8, 10] = float("inf"), float("nan"), top, -top
    got = ag.mx8_weight_grad(g, kept, dtype=F32).cpu()
    bad = torch.zeros(40, 100, dtype=torch.bool)
    bad[7:9] = True
    assert bool((~torch.isfinite(got))[bad].all())
    assert not bool(torch.isnan(got[9:]).any()) and bool(torch.isfinite(got[:7]).all()) and bool(torch.isfinite(got[11:]).all())
    zero = torch.zeros_like(g)
    zero[0] = 1
    spoilt = ag.Mx8(kept.codes, kept.scales.clone(), 100)
    spoilt.scales[3, 1] = 255                               # a block of NaN: its 32 columns
    got = ag.mx8_weight_grad(zero, spoilt, dtype=F32).cpu()
    bad = torch.zeros(40, 100, dtype=torch.bool)
    bad[:, 32:64] = True
    assert torch.equal(torch.isnan(got), bad)


def test_small_kept_values(ag):
    """Blocks whose values are subnormal numbers of bfloat16."""
    x = rows_of(64, 64) * 2.0 ** -124
    kept = ag.mx8_quantize(x)
    g = torch.full((64, 16), 2.0 ** 40, dtype=BF16, device="cuda")
    W, eW, _, _ = ref.weight_grad(g, ref.mx8_values(kept.codes, kept.scales, 64))
    within(ag.mx8_weight_grad(g, kept, dtype=F32), W, eW)


def test_another_stream_and_replayed_graph(ag):
    g, x = rows_of(900, 200, BF16), rows_of(900, 320, BF16)

    def step():
        y, kept = ag.mx8_activation(x, "silu", gated=True)
        dx = ag.mx8_activation_grad(y, kept, "silu", gated=True)
        return (y, dx) + ag.mx8_weight_grad(g, kept, bias=True, dtype=F32)
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, kept = ag.mx8_activation(x, "silu", gated=True, stream=s)
    dx = ag.mx8_activation_grad(y, kept, "silu", gated=True, stream=s)
    got = (y, dx) + ag.mx8_weight_grad(g, kept, bias=True, dtype=F32, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for seed in (11, 12, 13):
        x.copy_(rows_of(900, 320, BF16, seed))
        g.copy_(rows_of(900, 200, BF16, seed + 20))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("M,N,K", [(70000, 31, 64), (2100, 1001, 40), (300, 130, 1100), (4200, 515, 300)])
def test_gradients_cut_by_a_pass_of_their_own(ag, dtype, M, N, K):
    """Enough work for it, or a wide layer: rows at odd addresses, a last piece that the row's end cuts, and padding
    columns of the planes that hold no row's values."""
    check_wgrad(ag, M, N, K, dtype, F32)
    wide = rows_of(M, N + 3, dtype, seed=9)
    kept = ag.mx8_quantize(rows_of(M, K, seed=10))
    want = ag.mx8_weight_grad(wide[:, 1:1 + N].contiguous(), kept, bias=True, dtype=F32)
    got = ag.mx8_weight_grad(wide[:, 1:1 + N], kept, bias=True, dtype=F32)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("N", [1, 3, 7, 8, 9])
@pytest.mark.parametrize("dtype", FLOATS)
def test_narrow_gradients(ag, N, dtype):
    """Fewer columns than a piece of 8, at the end of their memory."""
    for M, K in ((1, 40), (33, 100), (400, 1030)):
        check_wgrad(ag, M, N, K, dtype, F32)


def test_rows_of_a_part_that_has_none(ag):
    """Parts are whole steps of 32 rows: the last parts may be empty, or hold one row; so may the bias gradient's."""
    for M in (32 * 4 * 3 + 1, 32 * 40 + 1, 32 * 33, 65 * 32 + 31):
        for N, K in ((8, 64), (47, 256)):
            check_wgrad(ag, M, N, K, BF16, F32)


def test_a_nan_in_the_last_row_stays_in_its_row(ag):
    """Rows behind the last one are zeros, not copies of it."""
    for dtype in FLOATS:
        for M, N, K in ((33, 16, 64), (2000, 1050, 64), (65, 24, 96)):
            g = torch.ones(M, N, dtype=dtype, device="cuda")
            g[M - 1, 3] = float("inf")
            got = ag.mx8_weight_grad(g, ag.mx8_quantize(torch.ones(M, K, device="cuda")), dtype=F32)
            assert bool((got[3] == float("inf")).all())
            got[3] = M
            assert bool((got == M).all())
