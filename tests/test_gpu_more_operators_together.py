"""The 8-bit operators and the policy loss as a program runs them: a training step of a gated layer and a head with
everything kept in 8 bits, each stage against its definition in 64 bits on what the stage before has left; the step in a
replayed graph; the trained layers served; and the example."""
import pytest
import torch

from tests import more_operators_ref as ref
from tests.operators_ref import within

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def ag():
    import paper_2601_01473_amd as m
    return m


def data(n, dim, hidden, classes, dtype, seed=1):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, dim, generator=g)
    w1, w2 = torch.randn(2 * hidden, dim, generator=g) / dim ** 0.5, torch.randn(classes, hidden, generator=g) / hidden ** 0.5
    y = torch.randint(-1, classes, (n,), generator=g)
    A, w = torch.randn(n, generator=g), torch.rand(n, generator=g) / n
    w[::5] = 0
    return [t.cuda() for t in (x.to(dtype), w1.to(dtype), w2.to(dtype), y, A, w)]


def step(ag, x, w1, w2, y, A, w, old, away):
    kept_x = ag.mx8_quantize(x)
    h = x @ w1.T
    a, kept_h = ag.mx8_activation(h, "gelu", gated=True)
    kept_a = ag.mx8_quantize(a)
    z = a @ w2.T
    loss, logp, dz = ag.policy_loss_grad(z, y, A, old, ref_logp=away, weight=w, kl=0.1)
    dw2, db2 = ag.mx8_weight_grad(dz, kept_a, bias=True, dtype=F32)
    da = dz @ w2
    dh = ag.mx8_activation_grad(da, kept_h, "gelu", gated=True)
    dw1, db1 = ag.mx8_weight_grad(dh, kept_x, bias=True, dtype=F32)
    return dict(kept_x=kept_x, h=h, a=a, kept_h=kept_h, kept_a=kept_a, z=z, loss=loss, logp=logp, dz=dz, dw2=dw2, db2=db2,
                da=da, dh=dh, dw1=dw1, db1=db1)


@pytest.mark.parametrize("n,dim,hidden,classes", [(64, 33, 20, 7), (300, 64, 96, 47), (1000, 100, 50, 300)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_training_step(ag, n, dim, hidden, classes, dtype):
    x, w1, w2, y, A, w = data(n, dim, hidden, classes, dtype)
    away = ag.policy_logprob(ag.mx8_activation(x @ w1.T, "gelu", gated=True, keep=False)[0] @ w2.T, y)
    old = away + 0.2 * torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    r = step(ag, x, w1, w2, y, A, w, old, away)
    value = lambda q: ref.mx8_values(q.codes, q.scales, q.cols)  # noqa: E731
    for q, t in ((r["kept_x"], x), (r["kept_h"], r["h"]), (r["kept_a"], r["a"])):
        codes, scales = ref.mx8(t)
        assert torch.equal(q.codes.cpu(), codes) and torch.equal(q.scales.cpu(), scales)
    within(r["a"], *ref.activation("gelu", r["h"], True), "a")
    L, eL, P, eP, G, eG = ref.policy(r["z"], y, A, old, away, w, kl=0.1)
    within(r["loss"], L, eL, "loss")
    within(r["logp"], P, eP, "logp")
    within(r["dz"], G, eG, "dz")
    within(r["dh"], *ref.activation_grad("gelu", r["da"], value(r["kept_h"]), True), "dh")
    for dw, db, g, q in ((r["dw2"], r["db2"], r["dz"], r["kept_a"]), (r["dw1"], r["db1"], r["dh"], r["kept_x"])):
        W, eW, b, eb = ref.weight_grad(g, value(q))
        within(dw, W, eW, "weight gradient")
        within(db, b, eb, "bias gradient")


def test_step_in_a_replayed_graph_beside_eager_steps(ag):
    n = 500
    args = data(n, 64, 96, 1000, BF16)
    old, away = torch.full((n,), -6.9, device="cuda"), torch.full((n,), -7.0, device="cuda")
    step(ag, *args, old, away)                              # library handles exist before the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(ag, *args, old, away)
    names = ("a", "loss", "logp", "dz", "dw2", "db2", "dh", "dw1", "db1")
    for seed in (5, 6, 7):
        for t, new in zip(args, data(n, 64, 96, 1000, BF16, seed)):
            t.copy_(new)
        graph.replay()
        eager = step(ag, *args, old, away)
        torch.cuda.synchronize()
        for k in names:
            assert torch.equal(out[k], eager[k]), k


def test_two_graphs_replayed_in_turn(ag):
    """Workspaces are the graphs' own: replays of two graphs that were captured one after the other do not disturb
    each other."""
    g, q = torch.randn(3000, 96, device="cuda"), ag.mx8_quantize(torch.randn(3000, 200, device="cuda"))
    x, w = torch.randn(60, 3000, device="cuda", dtype=BF16), ag.int8_quantize(torch.randn(300, 3000, device="cuda"))
    z, y, v = torch.randn(3, 60000, device="cuda"), torch.tensor([5, 59999, 0], device="cuda"), torch.ones(3, device="cuda")
    calls = [lambda: ag.mx8_weight_grad(g, q, bias=True), lambda: (ag.int8_linear(x, w),), lambda: ag.policy_loss_grad(z, y, v, -v)]
    want = [[t.clone() for t in c()] for c in calls]
    graphs, outs = [], []
    for c in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(c())
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        for t, u in zip(a, b):
            assert torch.equal(t, u)


def test_calls_on_two_streams_at_once(ag):
    g, q = torch.randn(20000, 64, device="cuda", dtype=BF16), ag.mx8_quantize(torch.randn(20000, 512, device="cuda"))
    x, w = torch.randn(64, 8192, device="cuda", dtype=BF16), ag.int8_quantize(torch.randn(1000, 8192, device="cuda"))
    want = ag.mx8_weight_grad(g, q, bias=True) + (ag.int8_linear(x, w),)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (a, b):
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        for s in (a, b):
            got.append(ag.mx8_weight_grad(g, q, bias=True, stream=s) + (ag.int8_linear(x, w, stream=s),))
    torch.cuda.synchronize()
    for r in got:
        for t, u in zip(r, want):
            assert torch.equal(t, u)


def test_served_layers(ag):
    """Two layers in 8 bits, as training leaves their weights."""
    x, w1, w2, *_ = data(70, 100, 64, 47, BF16)
    q1, q2 = ag.int8_quantize(w1), ag.int8_quantize(w2)
    h = ag.int8_linear(x, q1, dtype=F32)
    within(h, *ref.int8_product(*ref.int8(x), q1.codes, q1.scales, 100, None, False))
    a, _ = ag.mx8_activation(h, "gelu", gated=True, keep=False, dtype=BF16)
    z = ag.int8_linear(a, q2, torch.ones(47, device="cuda"), dtype=F32)
    within(z, *ref.int8_product(*ref.int8(a), q2.codes, q2.scales, 64, torch.ones(47), False))


SMALL = ["--scale", "10", "--dim", "40", "--hidden", "48", "--classes", "9", "--minibatches", "4", "--targets", "50",
         "--fanout", "5", "--steps", "6"]


def test_policy_nodes():
    from examples import policy_nodes
    r = policy_nodes.main(SMALL)
    assert all(v == v and abs(v) < 1e6 for v in r.values()), r
    # an element is off by at most half of 1/127 of its row's largest, which is below 6 times a row's mean size
    # here: 1.4 % of that size for each of a product's operands, two layers, errors that add up in no order
    assert 0 < r["error_8bit"] < 0.1


def test_policy_nodes_two_runs_agree():
    from examples import policy_nodes
    assert policy_nodes.main(SMALL) == policy_nodes.main(SMALL)


def test_offsets_beyond_32_bits(ag):
    """Matrices of more than 2^31 elements: the last rows are what they are alone, and a sum over all rows has them.
    (Few rows of logits take another kernel than many, which sums in another order, so these are held against the
    definition.)"""
    R, C, tail = 33000, 66000, 200
    z = torch.randn(64, C, device="cuda", dtype=BF16).repeat(-(-R // 64), 1)[:R]
    z[-tail:] = torch.randn(tail, C, device="cuda", dtype=BF16)
    last = z[-tail:].clone()
    y = torch.arange(R, device="cuda") % C
    v = torch.linspace(-1, 1, R, device="cuda")
    loss, logp, grad = ag.policy_loss_grad(z, y, v, -11 + v)
    for rows in (slice(0, 2), slice(R - 2, R)):
        L, eL, P, eP, G, eG = ref.policy(z[rows], y[rows], v[rows], -11 + v[rows])
        within(loss[rows], L, eL, "loss")
        within(logp[rows], P, eP, "logp")
        within(grad[rows], G, eG, "gradient")
    del loss, logp, grad
    for quantize, dequantize in ((ag.int8_quantize, ag.int8_dequantize), (ag.mx8_quantize, ag.mx8_dequantize)):
        q, want = quantize(z), quantize(last)
        assert torch.equal(q.codes[-tail:], want.codes) and torch.equal(q.scales[-tail:], want.scales)
        back = dequantize(q, BF16)
        assert torch.equal(back[-tail:], dequantize(want, BF16))
        del back
    # q: the kept rows.  Gradients that are zero but in the last rows leave their sum alone.
    g = torch.zeros(R, 8, device="cuda", dtype=BF16)
    g[-tail:] = torch.randn(tail, 8, device="cuda", dtype=BF16)
    v = ref.mx8_values(want.codes, want.scales, C)
    for dtype in (BF16, F32):
        W, eW, b, eb = ref.weight_grad(g[-tail:].to(dtype), v)
        dw, db = ag.mx8_weight_grad(g.to(dtype), q, bias=True, dtype=F32)
        # a sum over R rows, of which all but the last are zeros
        within(dw, W, eW * 4)
        within(db, b, eb * 4)
    y, kept = ag.mx8_activation(z, "silu")
    small, small_kept = ag.mx8_activation(last, "silu")
    assert torch.equal(y[-tail:], small) and torch.equal(kept.codes[-tail:], small_kept.codes)
    del y
    dx = ag.mx8_activation_grad(z, kept, "silu")
    assert torch.equal(dx[-tail:], ag.mx8_activation_grad(last, small_kept, "silu"))
