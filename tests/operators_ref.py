"""The operators' definitions in 64 bits on the CPU, with bounds on the error of float32 arithmetic.

Only tests import this module.  u = 2^-24 is float32's unit roundoff; rounding
to a result type costs its own (2^-24, 2^-11, 2^-8 for float32, float16,
bfloat16: half a unit in the last place, relative), or half the spacing of its
subnormals.
"""
import math

import torch

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
FLOATS = [torch.float32, torch.float16, torch.bfloat16]


def within(got, ref, err, what=""):
    """Every element of got within err of ref, plus one rounding to got's type."""
    g, r = got.detach().cpu().double(), ref
    assert g.shape == r.shape, (what, g.shape, r.shape)
    bound = err + ROUND[got.dtype] * (r.abs() + err) + TINY[got.dtype]
    same = (g == r) | (torch.isnan(g) & torch.isnan(r))
    # beyond the type's range the rounded value is infinite
    top = torch.finfo(got.dtype).max
    same |= torch.isinf(g) & (r.abs() + err >= top * (1 - ROUND[got.dtype])) & (torch.sign(g) == torch.sign(r))
    bad = ~same & ~((g - r).abs() <= bound)
    if bool(bad.any()):
        at = bad.nonzero()[0].tolist()
        raise AssertionError("%s: %d of %d off; at %s got %r, expected %r, bound %r"
                             % (what, int(bad.sum()), bad.numel(), at, float(g[tuple(at)]), float(r[tuple(at)]),
                                float(bound[tuple(at)] if bound.shape == r.shape else bound)))


# ----------------------------------------------------------------- embedding

def lookup(table, ids, scale):
    """(values, error): one float32 product per element."""
    t, i = table.cpu().double(), ids.cpu().long().reshape(-1)
    named = (i >= 0) & (i < len(t))
    out = torch.zeros(len(i), t.shape[1], dtype=torch.float64)
    out[named] = t[i[named]] * float(torch.tensor(scale, dtype=torch.float32))
    return out, U * out.abs()


def grad(grad_out, ids, num_rows, scale):
    """(distinct ids, rows, error): a float32 sum of m terms in any order is off by at most m u times the sum of their
    magnitudes; the product with the scale adds one rounding."""
    g, i = grad_out.cpu().double().reshape(ids.numel(), -1), ids.cpu().long().reshape(-1)
    named = (i >= 0) & (i < num_rows)
    names, which = torch.unique(i[named], return_inverse=True)
    s = float(torch.tensor(scale, dtype=torch.float32))
    rows = torch.zeros(len(names), g.shape[1], dtype=torch.float64)
    size = torch.zeros_like(rows)
    rows.index_add_(0, which, g[named])
    size.index_add_(0, which, g[named].abs())
    m = torch.bincount(which, minlength=len(names)).double().unsqueeze(1)
    return names, rows * s, (m + 2) * U * size * abs(s)


# ----------------------------------------------------------------- distillation

def distill(z, t, cls, labels=None, weight=None, temperature=1.0, soft=1.0, hard=0.0):
    """(loss, its error, gradient, its error), row by row from the definition.

    Error terms: d = (z - m) / T carries 3 u |d|; an exponential of it 4 u (|d| + 1) relative, |d| below 104 where it
    is not zero; a sum of C of them, each lane's terms one after the other, at most (C / 64 + 40) u relative.  So every
    probability is off by at most 2 delta relative and every logarithm of a sum by 2 delta, with
    delta = u (C / 64 + 40 + 8 D), D = the largest |d| that counts."""
    z, t, cls = z.cpu().double(), t.cpu().double(), cls.cpu().long()
    n, C = z.shape
    T, a, b = (float(torch.tensor(v, dtype=torch.float32)) for v in (temperature, soft, hard))
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.cpu().double()
    y = torch.full((n,), -1) if labels is None else labels.cpu().long()
    loss, eloss = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    grad, egrad = torch.zeros(n, C, dtype=torch.float64), torch.zeros(n, C, dtype=torch.float64)
    inf = float("inf")
    for i in range(n):
        if w[i] == 0:
            continue
        ok = (cls[i] >= 0) & (cls[i] < C)
        tt = t[i][ok] / T
        some = a > 0 and len(tt) > 0 and not bool((tt == -inf).all())
        named = b > 0 and 0 <= int(y[i]) < C
        m = z[i].max()
        if m == -inf:
            loss[i] = w[i] * inf if some or named else 0.0
            continue
        d = (z[i] - m) / T
        D = min(104.0, float(d[torch.isfinite(d)].abs().max()) if bool(torch.isfinite(d).any()) else 0.0)
        D = max(D, min(104.0, D * T))
        ln_q = d - torch.log(torch.exp(d).sum())
        q = torch.exp(ln_q)
        delta = U * (C / 64 + 40 + 8 * D)
        L, eL = torch.zeros((), dtype=torch.float64), 0.0
        if some:
            x = tt - tt.max()
            delta = max(delta, U * (len(tt) / 64 + 40 + 8 * min(104.0, float(x[torch.isfinite(x)].abs().max()))
                                    if bool(torch.isfinite(x).any()) else delta))
            p = torch.exp(x) / torch.exp(x).sum()
            ln_p = x - torch.log(torch.exp(x).sum())
            at = cls[i][ok]
            counts = p > 2.0 ** -149
            terms = p[counts] * (ln_p[counts] - ln_q[at[counts]])
            L = L + a * T * T * terms.sum()
            eL += a * T * T * float((p[counts] * (ln_p[counts].abs() + ln_q[at[counts]].abs() + 1)).sum()) * 4 * delta
            # a term below float32's range may be left out
            eL += a * T * T * 2.0 ** -120
            full = torch.zeros(C, dtype=torch.float64)
            full.index_add_(0, at, p)
            grad[i] += a * T * (q - full)
            egrad[i] += a * T * (q + full) * 4 * delta
        if named:
            d1 = z[i] - m
            ls = torch.log(torch.exp(d1).sum())
            L = L + b * (ls - d1[y[i]])
            eL += b * (1 + abs(float(ls)) + (abs(float(d1[y[i]])) if bool(torch.isfinite(d1[y[i]])) else 0)) * 4 * delta
            s = torch.exp(d1 - ls)
            one = torch.zeros(C, dtype=torch.float64)
            one[y[i]] = 1
            grad[i] += b * (s - one)
            egrad[i] += b * (s + one) * 4 * delta
        loss[i], eloss[i] = w[i] * L, abs(float(w[i])) * eL
        grad[i] *= w[i]
        egrad[i] = egrad[i] * abs(float(w[i])) + 2.0 ** -126
    return loss, eloss, grad, egrad


# ----------------------------------------------------------------- 4-bit rows

MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def mx4_block(values):
    """(scale code, 32 four-bit codes) of one block, element by element."""
    v = [float(x) for x in values] + [0.0] * (32 - len(values))
    if any(math.isnan(x) or math.isinf(x) for x in v):
        return 255, [0] * 32
    top = max(abs(x) for x in v)
    e = -127 if top == 0 else max(-127, math.frexp(top)[1] - 1 - 2)
    codes = []
    for x in v:
        mag = abs(x) / 2.0 ** e
        near = min(range(8), key=lambda c: (abs(mag - MAGNITUDES[c]), c & 1))
        codes.append(near + (8 if x < 0 else 0))
    return e + 127, codes


def mx4(x):
    """(codes, scales) of rows x as lists packed like the library's."""
    R, K = x.shape
    blocks = -(-K // 32)
    codes = torch.zeros(R, 16 * blocks, dtype=torch.uint8)
    scales = torch.zeros(R, blocks, dtype=torch.uint8)
    x = x.cpu().double()
    for r in range(R):
        for b in range(blocks):
            s, c = mx4_block(x[r, 32 * b:32 * b + 32].tolist())
            scales[r, b] = s
            for i in range(16):
                codes[r, 16 * b + i] = c[2 * i] | c[2 * i + 1] << 4
    return codes, scales


def mx4_values(codes, scales, cols):
    """The float64 values that codes and scales stand for."""
    codes, scales = codes.cpu(), scales.cpu()
    table = torch.tensor(MAGNITUDES + [-m for m in MAGNITUDES], dtype=torch.float64)
    v = table[torch.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1).long()]
    s = torch.exp2(scales.double() - 127)
    s[scales == 255] = float("nan")
    return (v * s.repeat_interleave(32, 1))[:, :cols]


def product(x, w, bias, relu):
    """(values, error) of x w^T + bias for float64 operands that are exact in float32: at most K + 1 additions, each off
    by at most 2^-23 (rounded or cut off)."""
    y = x @ w.T
    size = x.abs() @ w.abs().T
    if bias is not None:
        y, size = y + bias.cpu().double(), size + bias.cpu().double().abs()
    err = (x.shape[1] + 1) * 2.0 ** -23 * size
    return (torch.where(y < 0, 0.0, y) if relu else y), err
