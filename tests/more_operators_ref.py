"""The definitions of the 8-bit operators and of the policy loss in 64 bits on the CPU, with bounds on the error of
float32 arithmetic.  Only tests import this module; U, within and the result types' roundings are operators_ref's."""
import math

import torch

from tests.operators_ref import U, within  # noqa: F401

INF = float("inf")


def f32(v):
    return float(torch.tensor(v, dtype=torch.float32))


# ----------------------------------------------------------------- policy loss

def policy(z, actions, advantage, old, ref=None, weight=None, temperature=1.0, clip_low=0.2, clip_high=0.2, kl=0.0):
    """(loss, its error, logp, its error, gradient, its error), row by row from the definition.

    Error terms: d = (z - m) / T carries 3 u |d|; an exponential of it 4 u (|d| + 1) relative, |d| below 104 where it is
    not zero; a sum of C of them, each lane's terms one after the other, at most (C / 64 + 40) u relative.  So S, every
    probability and logp (absolutely) are off by at most 2 delta, delta = u (C / 64 + 40 + 8 D), D = the largest |d| that
    counts.  What follows from logp is computed in 64 bits, so it moves with logp alone: r by 2 delta relative, the
    loss by its slope, the slope by |r A| + kl e^d.  A row whose ratio lies within that of a border may be taken either way."""
    z, y = z.cpu().double(), actions.cpu().long()
    A, old = advantage.cpu().double(), old.cpu().double()
    n, C = z.shape
    T, low, high, b = f32(temperature), 1.0 - f32(clip_low), 1.0 + f32(clip_high), f32(kl)
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.cpu().double()
    out = [torch.zeros(n, dtype=torch.float64) for _ in range(4)]
    loss, eloss, logp, elogp = out
    grad, egrad = torch.zeros(n, C, dtype=torch.float64), torch.zeros(n, C, dtype=torch.float64)
    for i in range(n):
        if w[i] == 0 or not 0 <= int(y[i]) < C:
            continue
        if bool(torch.isnan(z[i]).any()) or bool((z[i] == INF).any()):
            loss[i] = logp[i] = float("nan")
            grad[i] = float("nan")
            continue
        a = float(A[i])
        if z[i, y[i]] == -INF:
            logp[i] = -INF
            loss[i] = w[i] * ((-low * a if a < 0 else 0.0) + (INF if b else 0.0))
            eloss[i] = 4 * U * abs(float(w[i] * a))
            continue
        d = (z[i] - z[i].max()) / T
        D = min(104.0, float(d[torch.isfinite(d)].abs().max()))
        delta = 2 * U * (C / 64 + 40 + 8 * D)
        ln_q = d - torch.log(torch.exp(d).sum())
        q = torch.exp(ln_q)
        lp = float(ln_q[y[i]])
        r = math.exp(lp - float(old[i]))
        free, held = r * a, min(max(r, low), high) * a
        value = -min(free, held) if a else 0.0
        slope = -free if a and free <= held else 0.0
        curve = abs(free) if a else 0.0
        eslope = curve * 1.1 * delta
        near = min(abs(r - low), abs(r - high)) <= 2 * delta * r
        evalue = curve * 1.1 * delta
        if b:
            away = float(ref[i]) - lp
            value += b * (math.expm1(away) - away)
            slope -= b * math.expm1(away)
            evalue += b * (abs(math.expm1(away)) * delta + math.exp(away) * delta * delta)
            eslope += b * math.exp(away) * 1.1 * delta
        if near:
            eslope += curve
        wi = float(w[i])
        logp[i], elogp[i] = lp, delta
        loss[i], eloss[i] = wi * value, abs(wi) * evalue
        one = torch.zeros(C, dtype=torch.float64)
        one[y[i]] = 1
        grad[i] = wi * slope / T * (one - q)
        g, eg = abs(wi * slope / T), abs(wi / T) * eslope + 4 * U * abs(wi * slope / T)
        egrad[i] = g * (q * 4 * delta + 4 * U * one) + eg * (one + q) + 2.0 ** -126
    return loss, eloss, logp, elogp, grad, egrad


# ----------------------------------------------------------------- 8-bit rows

def _nearest(n):
    """Whole numbers nearest to n (float64), ties to even."""
    low = torch.floor(n)
    part = n - low
    return low + ((part > 0.5) | ((part == 0.5) & (low % 2 == 1))).double()


def int8(x):
    """(codes int8 [R, 16 ceil(K / 16)], scales float32 [R]).  The quotient of two float32 numbers is not within a
    float64's rounding of a half without being one, so float64 decides as the exact quotient does."""
    R, K = x.shape
    x = x.cpu().double()
    codes = torch.zeros(R, -(-K // 16) * 16, dtype=torch.int8)
    scales = torch.zeros(R, dtype=torch.float32)
    for i in range(R):
        if K == 0:
            continue
        if not bool(torch.isfinite(x[i]).all()):
            scales[i] = float("nan")
            continue
        scales[i] = (x[i].abs().max() * f32(1 / 127)).float()      # the product of two float32 is exact in float64
        s = float(scales[i])
        if s > 0:
            codes[i, :K] = _nearest(x[i] / s).clamp(-127, 127).to(torch.int8)
    return codes, scales


def int8_values(codes, scales, cols):
    return codes.cpu()[:, :cols].double() * scales.cpu().double().unsqueeze(1)


def int8_product(xc, xs, wc, ws, cols, bias, relu):
    """(values, error): the whole sums are exact; then the conversion, two products and an addition round once each."""
    y = xc.cpu()[:, :cols].double() @ wc.cpu()[:, :cols].double().T
    y = y * xs.cpu().double().unsqueeze(1) * ws.cpu().double()
    err = 3 * U * y.abs()
    if bias is not None:
        y = y + bias.cpu().double()
        err = err + U * (y.abs() + err)
    err = err + 2.0 ** -149
    return (torch.where(y < 0, 0.0, y) if relu else y), err


# ----------------------------------------------------------------- 8-bit checkpoints

def mx8(x):
    """(codes int8 [R, 32 ceil(K / 32)], scales uint8 [R, ceil(K / 32)])."""
    R, K = x.shape
    blocks = -(-K // 32)
    wide = torch.zeros(R, 32 * blocks, dtype=torch.float64)
    wide[:, :K] = x.cpu().double()
    v = wide.view(R, blocks, 32)
    bad = ~torch.isfinite(v).all(2)
    top = torch.where(bad, 0.0, v.abs().amax(2) if v.numel() else torch.zeros(R, blocks, dtype=torch.float64))
    e = torch.where(top > 0, torch.frexp(top)[1] - 1, -127).clamp(min=-127)
    codes = _nearest(v * torch.exp2(6.0 - e.double()).unsqueeze(2)).clamp(-127, 127)
    codes[bad] = 0
    scales = torch.where(bad, 255, e + 127).to(torch.uint8)
    return codes.to(torch.int8).view(R, -1), scales


def mx8_values(codes, scales, cols):
    s = torch.exp2(scales.cpu().double() - 133)
    s[scales.cpu() == 255] = float("nan")
    return (codes.cpu().double() * s.repeat_interleave(32, 1))[:, :cols]


# The normal distribution in float32: a published rational form of erf is within 1.5e-7, Phi = (1 + erf) / 2 within
# half of that, and its few operations add less than 8 u.
PHI = 7.5e-8 + 8 * U


def act(kind, x):
    """(value, its error, slope, its error) at x (float64).  exp(-x) carries 2 u (|x| + 2) relative, which moves p = 1 /
    (1 + exp(-x)) by 1 - p times as much; 1 - p itself moves by p times as much.  The normal density's exponent x^2 / 2
    carries 2 u relative, so the density (x^2 + 6) u."""
    if kind == "silu":
        p, n = torch.sigmoid(x), torch.sigmoid(-x)
        ex = 2 * U * (x.abs() + 2)
        ep, en = p * (n * ex + 3 * U), n * (p * ex + 3 * U)
        # far below 0 the exponential overflows; what it gives there is below 2^-100
        slope = p * (1 + x * n)
        return x * p, (x * ep).abs() + U * (x * p).abs() + 2.0 ** -100, slope, \
            ep * (1 + x * n).abs() + p * (x * en).abs() + 6 * U * p * (1 + (x * n).abs()) + 2.0 ** -100
    phi = 0.5 * torch.erfc(-x / math.sqrt(2))
    dens = torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    slope = phi + x * dens
    return x * phi, x.abs() * PHI + U * (x * phi).abs() + 2.0 ** -126, slope, \
        PHI + (x * dens).abs() * (x * x + 8) * U + 2 * U * slope.abs() + 2.0 ** -126


def activation(kind, x, gated):
    """(y, its error)."""
    x = x.cpu().double()
    if not gated:
        v, e, _, _ = act(kind, x)
        return v, e
    a, b = x.chunk(2, 1)
    v, e, _, _ = act(kind, a)
    return v * b, e * b.abs() + 2 * U * (v * b).abs()


def activation_grad(kind, g, kept, gated):
    """(grad_x, its error) from the kept values (float64)."""
    g = g.cpu().double()
    if not gated:
        _, _, s, e = act(kind, kept)
        return g * s, g.abs() * e + 2 * U * (g * s).abs()
    a, b = kept.chunk(2, 1)
    v, ev, s, es = act(kind, a)
    return torch.cat([g * b * s, g * v], 1), \
        torch.cat([(g * b).abs() * es + 3 * U * (g * b * s).abs(), g.abs() * ev + 2 * U * (g * v).abs()], 1)


PIECES = {torch.bfloat16: 1, torch.float16: 2, torch.float32: 3}


def weight_grad(g, kept, old=None, old_bias=None):
    """(grad_weight, error, grad_bias, error): every product of a piece of g and a kept value is exact; at most pieces *
    M + 1024 additions, each off by at most 2^-23 (rounded or cut off), of terms that add up to at most (1 + 2^-6)
    of the magnitudes' sum."""
    pieces = PIECES[g.dtype]
    g = g.cpu().double()
    M = g.shape[0]
    y, size = g.T @ kept, g.abs().T @ kept.abs()
    b, bsize = g.sum(0), g.abs().sum(0)
    if old is not None:
        y, size = y + old.cpu().double(), size + old.cpu().double().abs()
    if old_bias is not None:
        b, bsize = b + old_bias.cpu().double(), bsize + old_bias.cpu().double().abs()
    return y, min(pieces * M + 1024, 4 * pieces * M + 4) * 2.0 ** -23 * 1.02 * size + 2.0 ** -133, b, (M + 4) * U * bsize
