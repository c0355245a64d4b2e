"""The clipped policy loss and its gradient on the GPU against the definition in 64 bits (tests/more_operators_ref.py)."""
import math

import pytest
import torch

from tests import more_operators_ref as ref
from tests.operators_ref import within

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
INF = float("inf")


@pytest.fixture(scope="module")
def ag():
    import paper_2601_01473_amd as m
    return m


def make(rows, C, dtype, idx=torch.int32, seed=1, spread=2.0, T=1.0):
    """(logits, actions, advantage, old, ref, weight), with padding, masked classes and rows of weight 0."""
    g = torch.Generator().manual_seed(seed)
    z = (spread * torch.randn(rows, C, generator=g)).to(dtype)
    z[1::4, (C + 1) // 2:] = -INF
    p = torch.softmax(z.double() / T, 1)
    y = torch.multinomial(p, 1, generator=g).squeeze(1) if rows else torch.zeros(0).long()
    logp = torch.log(p.gather(1, y.unsqueeze(1)).squeeze(1))
    old = (logp + 0.2 * torch.randn(rows, generator=g)).float()
    away = (logp + 0.4 * torch.randn(rows, generator=g)).float()
    A = torch.randn(rows, generator=g)
    A[3::7] = 0
    w = torch.rand(rows, generator=g)
    w[2::6] = 0
    y[4::9] = -100
    y[8::18] = C
    return z.cuda(), y.to(idx).cuda(), A.cuda(), old.cuda(), away.cuda(), w.cuda()


def check(ag, z, y, A, old, away=None, w=None, what="", **kw):
    """All four entry points against the definition; what they share agrees bit for bit."""
    more = dict(ref_logp=away, weight=w, **kw)
    L, eL, P, eP, G, eG = ref.policy(z, y, A, old, away, w, **kw)
    loss, logp, stats = ag.policy_loss(z, y, A, old, **more)
    within(loss, L, eL, what + " loss")
    within(logp, P, eP, what + " logp")
    grad = ag.policy_grad(z, y, A, old, stats, **more)
    within(grad, G, eG, what + " gradient")
    loss2, logp2, grad2 = ag.policy_loss_grad(z, y, A, old, **more)
    alone = ag.policy_logprob(z, y, weight=w, temperature=kw.get("temperature", 1.0))
    for a, b in ((loss, loss2), (logp, logp2), (grad, grad2), (logp, alone)):
        assert torch.equal(a.nan_to_num(nan=7.5), b.nan_to_num(nan=7.5)), what
    return loss, logp, grad


SIZES = [(1, 1), (1, 2), (3, 5), (64, 47), (33, 64), (7, 130), (5, 1000), (4, 1024), (3, 4097), (2, 9001), (2, 33000),
         (1, 100003), (3, 65536), (1, 140001), (600, 8200), (513, 2051)]


@pytest.mark.parametrize("rows,C", SIZES)
@pytest.mark.parametrize("dtype,idx", [(F32, torch.int32), (BF16, torch.int64), (F16, torch.int32)])
def test_sizes(ag, rows, C, dtype, idx):
    z, y, A, old, away, w = make(rows, C, dtype, idx)
    check(ag, z, y, A, old, away, w, kl=0.1)
    if rows < 100:
        z, y, A, old, away, w = make(rows, C, dtype, idx, seed=2, T=0.7)
        check(ag, z, y, A, old, temperature=0.7, clip_high=0.28)


@pytest.mark.parametrize("T", [0.25, 1.0, 3.0, 20.0])
@pytest.mark.parametrize("low,high,kl", [(0.2, 0.2, 0.0), (0.0, 0.0, 0.5), (1.0, 10.0, 0.02), (0.1, 0.3, 2.0)])
@pytest.mark.parametrize("C", [50, 700, 5000])
def test_terms_and_temperatures(ag, T, low, high, kl, C):
    z, y, A, old, away, w = make(19, C, F32, seed=3, T=T)
    check(ag, z, y, A, old, away if kl else None, w, temperature=T, clip_low=low, clip_high=high, kl=kl)
    check(ag, z, y, A, old, away, None, temperature=T, clip_low=low, clip_high=high, kl=kl)


@pytest.mark.parametrize("tz", [F32, F16, BF16])
@pytest.mark.parametrize("tg", [F32, F16, BF16])
@pytest.mark.parametrize("C", [90, 3000])
def test_every_pair_of_types(ag, tz, tg, C):
    z, y, A, old, away, w = make(6, C, tz, seed=4)
    more = dict(ref_logp=away, weight=w, kl=0.1)
    _, _, _, _, G, eG = ref.policy(z, y, A, old, away, w, kl=0.1)
    out = torch.empty(6, C, dtype=tg, device="cuda")
    _, _, got = ag.policy_loss_grad(z, y, A, old, out=out, **more)
    assert got is out
    within(out, G, eG)
    _, _, stats = ag.policy_loss(z, y, A, old, **more)
    out.zero_()
    ag.policy_grad(z, y, A, old, stats, out=out, **more)
    within(out, G, eG)


@pytest.mark.parametrize("C", [3, 60, 700, 5000, 140001])
def test_masked_infinite_and_undefined_logits(ag, C):
    z, y, A, old, away, w = make(12, C, F32, seed=5)
    y[:] = torch.arange(12, dtype=y.dtype) % C
    w[:] = 0.5
    A[:] = torch.tensor([1.0, -1.0] * 6)
    z[1::4] = torch.randn(3, C).cuda()
    low = torch.finfo(F32).min
    z[0] = -INF                                             # nothing is allowed
    z[1, int(y[1])] = -INF                                  # the action is not (A < 0)
    z[2, int(y[2])] = -INF                                  # the action is not (A > 0)
    z[3, 1:] = -INF                                         # one class is
    y[3] = 0
    z[4, 0] = float("nan")
    z[5, 1] = INF
    z[6, 1:] = low                                          # the type's lowest value in masked places
    y[6] = 0
    z[7] = low                                              # and everywhere
    w[8] = 0
    z[8] = float("nan")                                     # skipped
    y[9] = -1
    z[9] = INF                                              # padding
    A[4], A[10] = 0.0, 0.0                                  # an advantage of 0 does not hide a NaN
    old[11], old[10] = -INF, -INF
    A[11] = 1.0                                             # an infinite ratio, clipped
    for kl in (0.0, 0.3):
        # with T = 0.5 the lowest value divided by T is no float32
        for T in (1.0, 0.5):
            L, eL, P, eP, G, eG = ref.policy(z[:10], y[:10], A[:10], old[:10], away[:10], w[:10], temperature=T, kl=kl)
            loss, logp, grad = ag.policy_loss_grad(z, y, A, old, ref_logp=away, weight=w, temperature=T, kl=kl)
            within(loss[:10], L, eL, "loss")
            within(logp[:10], P, eP, "logp")
            within(grad[:10], G, eG, "gradient")
            assert bool(torch.isfinite(loss[10:]).all()) and bool(torch.isfinite(grad[10:]).all())
            if kl == 0.0:
                assert loss[10] == 0 and bool((grad[10:] == 0).all())
                assert float(loss[11]) == pytest.approx(-0.5 * 1.2, rel=1e-6)
            l2, p2, stats = ag.policy_loss(z, y, A, old, ref_logp=away, weight=w, temperature=T, kl=kl)
            g2 = ag.policy_grad(z, y, A, old, stats, ref_logp=away, weight=w, temperature=T, kl=kl)
            for a, b in ((loss, l2), (logp, p2), (grad, g2)):
                assert torch.equal(a.nan_to_num(nan=7.5), b.nan_to_num(nan=7.5))
    # NaN in what the row is compared with
    for name in range(3):
        args = [A.clone(), old.clone(), away.clone()]
        args[name][6] = float("nan")
        loss, logp, grad = ag.policy_loss_grad(z, y, args[0], args[1], ref_logp=args[2], weight=w, kl=0.3)
        assert bool(torch.isnan(loss[6])) and bool(torch.isfinite(logp[6])) and bool(torch.isnan(grad[6, 0]))
        assert not bool(torch.isnan(loss[7]))


def test_close_policies_keep_the_penalty_s_digits(ag):
    """exp d - d - 1 for d of 1e-4: 5e-9, of which float32 arithmetic would keep nothing."""
    z = torch.zeros(4, 8, device="cuda")
    y = torch.arange(4, device="cuda")
    lp = -math.log(8.0)
    old = torch.full((4,), lp, device="cuda")
    away = torch.tensor([lp - 3e-3, lp - 1e-3, lp + 1e-3, lp + 3e-3], device="cuda")
    zero = torch.zeros(4, device="cuda")
    loss, _, _ = ag.policy_loss_grad(z, y, zero, old, ref_logp=away, kl=1.0)
    d = away.cpu().double() - lp
    want = torch.expm1(d) - d
    # logp = -ln 8 is exact to 64 bits here: S = 8
    assert bool(((loss.cpu().double() - want).abs() <= 1e-6 * want).all()), (loss, want)


@pytest.mark.parametrize("C", [47, 3000])
def test_clipping_border(ag, C):
    """At the border itself the first term's slope is taken; a step beyond it is clipped."""
    z = torch.zeros(6, C, device="cuda")
    y = torch.zeros(6, dtype=torch.int64, device="cuda")
    lp = -math.log(C)
    high, low = math.log(1 + ref.f32(0.25)), math.log(1 - ref.f32(0.25))
    off = torch.tensor([high - 1e-4, high + 1e-4, high + 1e-4, low + 1e-4, low - 1e-4, low - 1e-4], dtype=torch.float64)
    old = (lp - off).float().cuda()
    A = torch.tensor([1.0, 1.0, -1.0, -1.0, -1.0, 1.0], device="cuda")
    _, _, grad = ag.policy_loss_grad(z, y, A, old, clip_low=0.25, clip_high=0.25)
    assert (grad[:, 0] != 0).tolist() == [True, False, True, True, False, True]
    # old = logp exactly where log C is, with clips of 0: the ratio is 1 and not clipped
    z = torch.zeros(2, 1, device="cuda")
    loss, logp, grad = ag.policy_loss_grad(z, y[:2], A[:2], torch.zeros(2, device="cuda"), clip_low=0.0, clip_high=0.0)
    assert loss.tolist() == [-1.0, -1.0] and logp.tolist() == [0.0, 0.0] and bool((grad == 0).all())


@pytest.mark.parametrize("C", [11, 129, 2600, 70001])
def test_strides_in_place_and_untouched_memory(ag, C):
    z, y, A, old, away, w = make(9, C, BF16, seed=6)
    wide = torch.full((9, C + 13), 3.0, dtype=BF16, device="cuda")
    wide[:, 5:5 + C] = z
    view = wide[:, 5:5 + C]
    want = ag.policy_loss_grad(z, y, A, old, ref_logp=away, weight=w, kl=0.2)
    out = torch.full((9, C + 7), 9.0, dtype=F32, device="cuda")
    got = ag.policy_loss_grad(view, y, A, old, ref_logp=away, weight=w, kl=0.2, out=out[:, 3:3 + C])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2].to(BF16), want[2])
    assert bool((out[:, :3] == 9).all()) and bool((out[:, 3 + C:] == 9).all())
    # the gradient over the logits, from either entry point
    _, _, stats = ag.policy_loss(view, y, A, old, ref_logp=away, weight=w, kl=0.2)
    second = wide.clone()
    ag.policy_loss_grad(view, y, A, old, ref_logp=away, weight=w, kl=0.2, out=view)
    v2 = second[:, 5:5 + C]
    ag.policy_grad(v2, y, A, old, stats, ref_logp=away, weight=w, kl=0.2, out=v2)
    assert torch.equal(view, want[2]) and torch.equal(v2, want[2])
    assert bool((wide[:, :5] == 3).all()) and bool((wide[:, 5 + C:] == 3).all())
    # one row of logits for all decisions
    one = z[:1].expand(9, C)
    check(ag, one, torch.where(y < C // 2, y, 0), A, old, away, w, kl=0.2)


@pytest.mark.parametrize("C", [64, 5000])
def test_no_rows_and_only_skipped_rows(ag, C):
    z, y, A, old, away, w = make(0, C, F32)
    loss, logp, grad = ag.policy_loss_grad(z, y, A, old)
    assert loss.numel() == logp.numel() == grad.numel() == 0
    z = torch.full((5, C), float("nan"), device="cuda")
    y = torch.full((5,), -1, dtype=torch.int32, device="cuda")
    v = torch.zeros(5, device="cuda")
    loss, logp, grad = ag.policy_loss_grad(z, y, v, v)
    assert bool((loss == 0).all()) and bool((logp == 0).all()) and bool((grad == 0).all())


def test_gradient_against_differences(ag):
    """Central differences of the float64 definition's loss, at rows well inside and outside the clip."""
    z, y, A, old, away, w = make(14, 9, F32, seed=8)
    kw = dict(temperature=1.3, kl=0.2)
    _, _, grad = ag.policy_loss_grad(z, y, A, old, ref_logp=away, weight=w, **kw)
    h = 1e-5
    zd = z.cpu().double()
    num = torch.zeros(14, 9, dtype=torch.float64)
    for j in range(9):
        up, down = zd.clone(), zd.clone()
        up[:, j] += h
        down[:, j] -= h
        num[:, j] = (ref.policy(up, y, A, old, away, w, **kw)[0] - ref.policy(down, y, A, old, away, w, **kw)[0]) / (2 * h)
    num.nan_to_num_(0.0)                                    # masked logits stay masked
    # a difference is off by h^2 / 6 of the third derivative (below 100 here) and 1e-16 / h of rounding
    assert float((grad.cpu().double() - num).abs().max()) < 1e-6


def test_another_stream_and_replayed_graph(ag):
    z, y, A, old, away, w = make(33, 3001, BF16, seed=9)
    want = ag.policy_loss_grad(z, y, A, old, ref_logp=away, weight=w, kl=0.1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ag.policy_loss_grad(z, y, A, old, ref_logp=away, weight=w, kl=0.1, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    long = make(2, 90001, BF16, seed=10)                    # with a workspace
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ag.policy_loss_grad(z, y, A, old, ref_logp=away, weight=w, kl=0.1)
        out2 = ag.policy_loss_grad(*long[:4], ref_logp=long[4], kl=0.1)
    for seed in (11, 12, 13):
        new, new2 = make(33, 3001, BF16, seed=seed), make(2, 90001, BF16, seed=seed)
        for t, n in zip((z, y, A, old, away, w) + long, new + new2):
            t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in ((out, ag.policy_loss_grad(z, y, A, old, ref_logp=away, weight=w, kl=0.1)),
                          (out2, ag.policy_loss_grad(*long[:4], ref_logp=long[4], kl=0.1))):
            for a, b in zip(got, want):
                assert torch.equal(a, b)


def test_many_rows_of_each_kernel(ag):
    """More rows than a grid holds at once; the same rows again give the same bits."""
    for rows, C, dtype in ((70001, 5, F32), (70001, 40, BF16), (3000, 1500, F16)):
        z, y, A, old, away, w = make(997, C, dtype, seed=14)
        n = -(-rows // 997)
        big = [t.repeat(n, *[1] * (t.dim() - 1))[:rows].contiguous() for t in (z, y, A, old, away, w)]
        few = check(ag, z, y, A, old, away, w, kl=0.1)
        got = ag.policy_loss_grad(*big[:4], ref_logp=big[4], weight=big[5], kl=0.1)
        for a, b in zip(got, few):
            assert torch.equal(a, b.repeat(n, *[1] * (b.dim() - 1))[:rows])


@pytest.mark.parametrize("C", [40, 3000, 100003])
@pytest.mark.parametrize("T", [1e-3, 1e30])
def test_extreme_temperatures(ag, C, T):
    """Masked classes stay masked where the factor log2(e) / T has no smaller part left, or is large."""
    z, y, A, old, away, w = make(5, C, F32, seed=15)
    if T < 1:
        y[:] = z.argmax(1)                                  # any other class has no probability left
        old[:] = -0.1
    check(ag, z, y, A, old, away, w, temperature=T, kl=0.0)
