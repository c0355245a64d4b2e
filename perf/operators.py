"""What the training and serving operators' speed is measured on.

Three operators that work beside the hyperbatch path, each on the arrays that
path hands over (node lists, target logits, feature rows):

  lookup    rows of a learned table for a list of ids, scaled
  grad      its gradient, summed over equal ids: as a dense table, or as the
            distinct rows alone ("rows", what a sparse optimiser step takes)
  distill   the loss of a student's logits against a teacher's top logits (with
            an optional label term), and its gradient: in one call ("step"), or
            the loss first and the gradient from its statistics ("split")
  quantize  rows to microscaled 4-bit floating point and back to values
  linear    rows times a 4-bit weight, the rows quantised on the way in

A state holds what a program has before the call: the table, the ids, the
gradient that arrives, the logits, the 4-bit weight.
"""
import math

import torch

own = False

_DT = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16,
       "int32": torch.int32, "int64": torch.int64}


def listed():
    return [
        # the targets of one minibatch of the smallest workload: latency alone
        _lookup("lookup 256 of 2^14 x 64", 1 << 14, 64, 256, "float32", "float32"),
        # every node of a hyperbatch on the middle workload's graph: float32
        # master rows, bf16 rows out for the forward
        _lookup("lookup 2000003 of 2^20 x 128", 1 << 20, 128, 2000003, "float32", "bfloat16", skew=2.0),
        # one minibatch's nodes, odd counts: sort, sums and empty rows in few launches
        _grad("grad 777 to 2^12 x 64", 1 << 12, 64, 777, "float32", skew=1.5),
        # a hyperbatch's nodes: hubs recur in every minibatch, most nodes once;
        # only the distinct rows are wanted
        _grad("grad rows 1500007 of 2^20 x 256", 1 << 20, 256, 1500007, "bfloat16", form="rows", skew=2.0),
        # tokens of long texts over a vocabulary of odd size: a few tokens take
        # a large share of all positions; the whole table's gradient
        _grad("grad 131072 to 50021 x 1024", 50021, 1024, 131072, "bfloat16", skew=6.0, ids="int64"),
        # node classes of the smallest workload's hyperbatch (8 x 256 targets)
        _distill("distill 2048 x 47", 2048, 47, 8, "float32", T=2.0, hard=0.3),
        # token logits of a training step over a large vocabulary
        _distill("distill 8192 x 65536", 8192, 65536, 64, "bfloat16", T=2.0, hard=0.5, idx="int64"),
        # few positions, an odd vocabulary (rows that are not 16-byte aligned),
        # gradient from the saved statistics
        _distill("distill split 8 x 100003", 8, 100003, 32, "float16", form="split"),
        # rows of odd length: the last block is partial
        _quantize("quantize 1000 x 1003", 1000, 1003, "float32"),
        # the hidden rows of a hyperbatch's targets at the widest layer allowed
        _quantize("quantize 65536 x 1024", 65536, 1024, "bfloat16"),
        # one row through a 4096 x 4096 layer: the weight is read once
        _linear("linear 1 x 4096 x 4096", 1, 4096, 4096, "bfloat16"),
        # many rows through a wide layer
        _linear("linear 8192 x 8192 x 8192", 8192, 8192, 8192, "bfloat16", relu=True),
    ]


def draw(rng):
    """One more case of the listed ones' ranges: 1 to 2M ids over tables of 64 to 2^21 rows of 1 to 2048 elements;
    1 to 65536 rows of 2 to 131072 logits with 1 to 128 teacher entries; 4-bit rows and layers of 1 to 8192 columns."""
    def spread(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    float_types = ["float32", "float16", "bfloat16", "bfloat16"]
    kind = rng.choice(["lookup", "grad", "grad", "grad", "distill", "distill", "distill", "quantize", "linear", "linear"])
    while True:
        if kind in ("lookup", "grad"):
            V, D, n = spread(64, 1 << 21), spread(1, 2048), spread(1, 2 << 20)
            if rng.random() < 0.4:
                D = 1 << (D.bit_length() - 1)
            if n * D > 1 << 28 or V * D > 1 << 28:
                continue
            skew, ids = rng.choice([1.0, 1.5, 2.0, 4.0, 6.0]), rng.choice(["int32", "int64"])
            if kind == "lookup":
                case = _lookup("", V, D, n, rng.choice(float_types), rng.choice(float_types), skew, ids)
            else:
                case = _grad("", V, D, n, rng.choice(float_types), rng.choice(["dense", "rows"]), skew, ids)
        elif kind == "distill":
            rows, C = spread(1, 65536), spread(2, 131072)
            if rng.random() < 0.4:
                C = -(-C // 8) * 8
            if rows * C > 1 << 28:
                continue
            case = _distill("", rows, C, min(C, spread(1, 128)), rng.choice(float_types),
                            T=rng.choice([1.0, 1.0, 2.0, 4.0]), hard=rng.choice([0.0, 0.3, 0.5]),
                            form=rng.choice(["step", "step", "split"]), idx=rng.choice(["int32", "int64"]))
        elif kind == "quantize":
            rows, cols = spread(1, 65536), spread(1, 8192)
            if rows * cols > 1 << 26:
                continue
            case = _quantize("", rows, cols, rng.choice(float_types))
        else:
            M, N, K = spread(1, 8192), spread(16, 8192), spread(32, 8192)
            if rng.random() < 0.5:
                N, K = -(-N // 32) * 32, -(-K // 32) * 32
            if rng.random() < 0.3:
                M = rng.randint(1, 16)
            case = _linear("", M, N, K, rng.choice(float_types), out=rng.choice(float_types),
                           relu=rng.random() < 0.3, bias=rng.random() < 0.7)
        del case["name"]
        return case


def _lookup(name, V, D, n, dtype, out, skew=1.0, ids="int32"):
    return dict(name=name, kind="lookup", V=V, D=D, n=n, dtype=dtype, out=out, skew=skew, ids=ids, scale=D ** 0.5)


def _grad(name, V, D, n, dtype, form="dense", skew=1.0, ids="int32"):
    return dict(name=name, kind="grad", V=V, D=D, n=n, dtype=dtype, form=form, skew=skew, ids=ids, scale=D ** 0.5)


def _distill(name, rows, C, k, dtype, T=1.0, hard=0.0, form="step", idx="int32"):
    return dict(name=name, kind="distill", rows=rows, C=C, k=k, dtype=dtype, T=T, hard=hard, form=form, idx=idx)


def _quantize(name, rows, cols, dtype):
    return dict(name=name, kind="quantize", rows=rows, cols=cols, dtype=dtype)


def _linear(name, M, N, K, dtype, out=None, relu=False, bias=True):
    return dict(name=name, kind="linear", M=M, N=N, K=K, dtype=dtype, out=out or dtype, relu=relu, bias=bias)


# ----------------------------------------------------------------- states

class _State:
    pass


def _ids(case, gen):
    """The case's ids: floor(V u^skew) for uniform u, one in 64 of them padding (-1).  Which ids occur, and how often,
    is the case's, so the number of distinct rows is too (a program has it from its batch's statistics); the seed
    gives their order."""
    own_gen = torch.Generator(device="cuda").manual_seed(case["V"] * 31 + case["n"])
    u = torch.rand(case["n"], device="cuda", generator=own_gen, dtype=torch.float64)
    ids = (case["V"] * u ** case["skew"]).long().clamp(max=case["V"] - 1)
    ids[1::64] = -1
    return ids[torch.randperm(case["n"], device="cuda", generator=gen)].to(_DT[case["ids"]])


def _distinct(ids):
    u = torch.unique(ids)
    return int((u >= 0).sum())


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    kind = case["kind"]
    if kind == "lookup":
        s.table = (normal(case["V"], case["D"]) / math.sqrt(case["D"])).to(_DT[case["dtype"]])
        s.ids = _ids(case, gen)
    elif kind == "grad":
        s.ids = _ids(case, gen)
        s.distinct = _distinct(s.ids)
        s.grad_out = (normal(case["n"], case["D"]) / 64).to(_DT[case["dtype"]])
    elif kind == "distill":
        rows, C, k = case["rows"], case["C"], case["k"]
        z = normal(rows, C).mul_(2)
        s.logits = z.to(_DT[case["dtype"]])
        t, c = z.add_(normal(rows, C)).topk(k, dim=1)
        del z
        s.teacher = t.to(torch.bfloat16 if case["dtype"] == "bfloat16" else torch.float32)
        # a fifth of the rows keep fewer entries, down to none
        keep = torch.randint(0, k + 1, (rows, 1), device="cuda", generator=gen)
        keep = torch.where(torch.rand(rows, 1, device="cuda", generator=gen) < 0.2, keep, k)
        s.classes = torch.where(torch.arange(k, device="cuda") < keep, c, -1).to(_DT[case["idx"]])
        s.labels = torch.randint(0, C, (rows,), device="cuda", generator=gen)
        s.labels[::17] = -1
        s.labels = s.labels.to(_DT[case["idx"]]) if case["hard"] else None
        s.weight = torch.rand(rows, device="cuda", generator=gen) / rows
        s.weight[5::32] = 0
    elif kind == "quantize":
        # rows of different scales, as activations have
        s.x = (normal(case["rows"], case["cols"]) * torch.exp(2 * normal(case["rows"], 1))).to(_DT[case["dtype"]])
    else:
        s.x = normal(case["M"], case["K"]).to(_DT[case["dtype"]])
        w = normal(case["N"], case["K"]) / math.sqrt(case["K"])
        s.codes, s.scales = _mx4_codes(w)
        s.bias = 0.1 * normal(case["N"]) if case["bias"] else None
    return s


# ----------------------------------------------------------------- plain forms

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx4_codes(x):
    """float32 [R, K] -> codes uint8 [R, 16 ceil(K / 32)] (element 2i in the low four bits) and scales uint8 [R, ceil(K / 32)]."""
    R, K = x.shape
    blocks = -(-K // 32)
    x = torch.nn.functional.pad(x, (0, 32 * blocks - K)).view(R, blocks, 32)
    top = (x.abs().amax(2).view(torch.int32) >> 23) & 255            # biased exponent of the block's largest value
    scales = torch.where(top == 255, 255, (top - 2).clamp(min=0))
    y = torch.ldexp(x, (127 - scales).unsqueeze(2))
    a = y.abs()
    # steps at the midpoints; a midpoint goes to the neighbour with the even code
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    code = (code + 8 * (x < 0)).to(torch.uint8).view(R, blocks * 16, 2)
    return code[..., 0] | (code[..., 1] << 4), scales.to(torch.uint8)


def _mx4_values(codes, scales, K):
    grid = torch.tensor(_GRID + tuple(-g for g in _GRID), device="cuda")
    R = codes.shape[0]
    v = grid[torch.stack([codes & 15, codes >> 4], 2).long()].view(R, -1, 32)
    return torch.ldexp(v, scales.int().unsqueeze(2) - 127).view(R, -1)[:, :K]


def _plain_grad(s):
    c = s.case
    valid = (s.ids >= 0) & (s.ids < c["V"])
    g = torch.where(valid.unsqueeze(1), s.grad_out.float(), 0.0)
    ids = s.ids.long().clamp(0, c["V"] - 1)
    if c["form"] == "dense":
        out = torch.zeros(c["V"], c["D"], device="cuda").index_add_(0, ids, g)
        return (out * c["scale"]).to(s.grad_out.dtype)
    count = torch.zeros(c["V"], dtype=torch.int32, device="cuda").index_add_(0, ids, valid.int())
    used = (count > 0).nonzero().squeeze(1)
    place = torch.cumsum(count > 0, 0) - 1
    rows = torch.zeros(s.distinct, c["D"], device="cuda").index_add_(0, place[ids].clamp(min=0), g)
    return used.int(), (rows * c["scale"]).to(s.grad_out.dtype)


def _plain_distill(s):
    c = s.case
    T, hard = c["T"], c["hard"]
    soft = 1.0 - hard
    z = s.logits.float()
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z / T)
    sums = e.sum(1, keepdim=True)
    valid = (s.classes >= 0) & (s.classes < c["C"])
    t = torch.where(valid, s.teacher.float() / T, float("-inf"))
    some = valid.any(1, keepdim=True)
    t = torch.where(some, t - t.amax(1, keepdim=True), 0.0)
    p = torch.where(some & valid, torch.exp(t), 0.0)
    ps = torch.where(some, p.sum(1, keepdim=True), 1.0)
    p = p / ps
    cls = torch.where(valid, s.classes.long(), 0)
    ln_q = z.gather(1, cls) / T - torch.log(sums)
    ln_p = t - torch.log(ps)
    loss = soft * T * T * torch.where(p > 0, p * (ln_p - ln_q), 0.0).sum(1)
    w = s.weight.unsqueeze(1)
    a = (soft * T) * w
    grad = e * (a * some / sums)
    grad.scatter_add_(1, cls, -a * p)
    if hard:
        named = ((s.labels >= 0) & (s.labels < c["C"])).unsqueeze(1)
        y = torch.where(named, s.labels.long().unsqueeze(1), 0)
        e1 = torch.exp(z)
        s1 = e1.sum(1, keepdim=True)
        loss = loss + hard * torch.where(named, torch.log(s1) - z.gather(1, y), 0.0).squeeze(1)
        b = hard * w * named
        grad += e1 * (b / s1)
        grad.scatter_add_(1, y, -b)
    return loss * s.weight, grad.to(s.logits.dtype)


def _plain(s):
    c = s.case
    if c["kind"] == "lookup":
        valid = (s.ids >= 0) & (s.ids < c["V"])
        rows = s.table[s.ids.long().clamp(0, c["V"] - 1)].float() * c["scale"]
        return torch.where(valid.unsqueeze(1), rows, 0.0).to(_DT[c["out"]])
    if c["kind"] == "grad":
        return _plain_grad(s)
    if c["kind"] == "distill":
        return _plain_distill(s)
    if c["kind"] == "quantize":
        return _mx4_values(*_mx4_codes(s.x.float()), c["cols"]).to(s.x.dtype)
    x = _mx4_values(*_mx4_codes(s.x.float()), c["K"])
    y = x @ _mx4_values(s.codes, s.scales, c["K"]).T
    if s.bias is not None:
        y = y + s.bias
    return (torch.where(y > 0, y, 0.0) if c["relu"] else y).to(_DT[c["out"]])


# ----------------------------------------------------------------- the framework's operators

def _own(s):
    import paper_2601_01473_amd as ag

    c = s.case
    if c["kind"] == "lookup":
        return ag.embedding_lookup(s.table, s.ids, scale=c["scale"], dtype=_DT[c["out"]])
    if c["kind"] == "grad" and c["form"] == "dense":
        return ag.embedding_grad(s.grad_out, s.ids, c["V"], scale=c["scale"])
    if c["kind"] == "grad":
        ids, rows, _ = ag.embedding_grad_rows(s.grad_out, s.ids, c["V"], s.distinct, scale=c["scale"])
        return ids, rows
    if c["kind"] == "distill":
        args = dict(labels=s.labels, weight=s.weight, temperature=c["T"], soft=1.0 - c["hard"], hard=c["hard"])
        if c["form"] == "step":
            return ag.distill_loss_grad(s.logits, s.teacher, s.classes, **args)
        loss, stats = ag.distill_loss(s.logits, s.teacher, s.classes, **args)
        return loss, ag.distill_grad(s.logits, s.teacher, s.classes, stats, **args)
    if c["kind"] == "quantize":
        return ag.mx4_dequantize(ag.mx4_quantize(s.x), dtype=s.x.dtype)
    return ag.mx4_linear(s.x, ag.Mx4(s.codes, s.scales, c["K"]), s.bias, relu=c["relu"], dtype=_DT[c["out"]])


def run(state):
    return _own(state) if own else _plain(state)


# ----------------------------------------------------------------- what is measured against

def work(case):
    """Each input once and each output once; a table's rows that no id names are not read."""
    size = {"float32": 4, "float16": 2, "bfloat16": 2, "int32": 4, "int64": 8}
    kind = case["kind"]
    if kind in ("lookup", "grad"):
        distinct = _distinct(_ids(case, torch.Generator(device="cuda").manual_seed(1)))
        n, D, s = case["n"], case["D"], size[case["dtype"]]
        if kind == "lookup":
            return dict(bytes=n * size[case["ids"]] + distinct * D * s + n * D * size[case["out"]], flops=n * D)
        out = case["V"] * D * s if case["form"] == "dense" else distinct * (4 + D * s)
        return dict(bytes=n * size[case["ids"]] + n * D * s + out, flops=n * D)
    if kind == "distill":
        rows, C, k = case["rows"], case["C"], case["k"]
        entries = rows * k * ((2 if case["dtype"] == "bfloat16" else 4) + size[case["idx"]])
        # per logit: difference, exponential, sum, and the product of the gradient; twice with a label term
        return dict(bytes=2 * rows * C * size[case["dtype"]] + entries + 8 * rows,
                    flops=rows * C * (8 if case["hard"] else 4))
    if kind == "quantize":
        return dict(bytes=2 * case["rows"] * case["cols"] * size[case["dtype"]], flops=4 * case["rows"] * case["cols"])
    M, N, K = case["M"], case["N"], case["K"]
    blocks = -(-K // 32)
    return dict(bytes=M * K * size[case["dtype"]] + N * blocks * 17 + M * N * size[case["out"]] + 4 * N,
                flops=2 * M * N * K)


# The definitions in 64 bits.

def _exact_mx4(x):
    """The values that rows x (float64) stand for in microscaled 4-bit floating point, by the definition: a block of 32
    has the scale 2^(floor(log2 max|x|) - 2), an element the nearest of the eight magnitudes, ties to an even code."""
    R, K = x.shape
    out = torch.empty_like(x)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    order = [0, 2, 4, 6, 1, 3, 5, 7]              # even codes first: the first of two equally near ones is kept
    step = max(1, (1 << 26) // max(K, 1))
    for r in range(0, R, step):
        part = x[r:r + step]
        wide = torch.zeros(part.shape[0], -(-K // 32) * 32, dtype=torch.float64, device=x.device)
        wide[:, :K] = part
        b = wide.view(part.shape[0], -1, 32)
        m = b.abs().max(dim=2, keepdim=True).values
        _, e = torch.frexp(m)                      # m = f 2^e, f in [0.5, 1)
        scale = torch.exp2((e - 3).clamp(min=-127).double())
        mag = b.abs() / scale
        best = torch.full_like(mag, 100.0)
        got = torch.zeros_like(mag)
        for i in order:
            d = (mag - grid[i]).abs()
            got = torch.where(d < best, grid[i], got)
            best = torch.minimum(best, d)
        out[r:r + step] = (torch.sign(b) * got * scale).view(part.shape[0], -1)[:, :K]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "lookup":
        out = torch.zeros(case["n"], case["D"], dtype=torch.float64, device="cuda")
        named = (s.ids >= 0).nonzero().squeeze(1)
        out[named] = s.table.double()[s.ids[named].long()] * case["scale"]
        return out
    if kind == "grad":
        order = torch.argsort(s.ids, stable=True)
        order = order[s.ids[order] >= 0]
        names, lengths = torch.unique_consecutive(s.ids[order], return_counts=True)
        which = torch.repeat_interleave(torch.arange(len(names), device="cuda"), lengths)
        rows = torch.zeros(len(names), case["D"], dtype=torch.float64, device="cuda")
        rows.index_add_(0, which, s.grad_out.double()[order])
        rows *= case["scale"]
        if case["form"] == "rows":
            return names.int(), rows
        out = torch.zeros(case["V"], case["D"], dtype=torch.float64, device="cuda")
        out[names.long()] = rows
        return out
    if kind == "distill":
        losses, grads = [], []
        T, hard, C = case["T"], case["hard"], case["C"]
        step = max(1, (1 << 27) // C)
        for r in range(0, case["rows"], step):
            z = s.logits[r:r + step].double()
            n = z.shape[0]
            ln_q = torch.log_softmax(z / T, 1)
            p = torch.zeros_like(z)
            cls, t = s.classes[r:r + step].long(), s.teacher[r:r + step].double() / T
            t = t.masked_fill(cls < 0, float("-inf"))
            has = (cls >= 0).any(1)
            soft_p = torch.where(has[:, None], torch.softmax(t, 1), 0.0)
            at = torch.arange(n, device="cuda")[:, None].expand_as(cls)
            p.index_put_((at, cls.clamp(min=0)), torch.where(cls >= 0, soft_p, 0.0), accumulate=True)
            loss = (1 - hard) * T * T * torch.where(p > 0, p * (torch.log(p) - ln_q), 0.0).sum(1)
            grad = (1 - hard) * T * (torch.exp(ln_q) * has[:, None] - p)
            if hard:
                y = s.labels[r:r + step].long()
                ln_1 = torch.log_softmax(z, 1)
                named = (y >= 0).double()
                loss -= hard * named * ln_1[torch.arange(n, device="cuda"), y.clamp(min=0)]
                one = torch.exp(ln_1)
                one[torch.arange(n, device="cuda"), y.clamp(min=0)] -= 1
                grad += hard * named[:, None] * one
            w = s.weight[r:r + step].double()
            losses.append(loss * w)
            grads.append(grad * w[:, None])
        return torch.cat(losses), torch.cat(grads)
    if kind == "quantize":
        return _exact_mx4(s.x.double())
    codes = torch.stack([s.codes & 15, s.codes >> 4], 2).view(case["N"], -1).long()
    power, half = (codes >> 1) & 3, codes & 1      # sign, two bits of exponent, one of mantissa
    w = torch.where(power > 0, (1 + 0.5 * half) * torch.exp2(power.double() - 1), 0.5 * half)
    w = torch.where(codes >= 8, -w, w) * torch.exp2(s.scales.double() - 127).repeat_interleave(32, 1)
    y = _exact_mx4(s.x.double()) @ w[:, :case["K"]].T.contiguous()
    if s.bias is not None:
        y = y + s.bias.double()
    return y.clamp(min=0) if case["relu"] else y
