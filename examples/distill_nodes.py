"""A node classifier learnt from a teacher's top logits, then served in 4 bits.

    python examples/distill_nodes.py [--scale 14] [--dim 64] [--classes 47] [--steps 60]

Every node has a learned row; a target's representation is its own row plus the
mean of its sampled neighbours' rows, and a linear head gives its logits.  A
step is one hyperbatch:

    prepare             the targets' sampled neighbourhoods
    Batch.embedding     the rows of their nodes, float32 masters to bfloat16
    distill_loss_grad   loss against the teacher's top logits and the labels,
                        with the logits' gradient
    Batch.embedding_grad_rows   the gradient of the distinct nodes' rows alone,
                        which a sparse step then applies
    embedding_grad      sums of rows with equal ids, in a fixed order: the mean
                        over neighbours and its gradient

After training the head is laid out in 4 bits once (mx4_quantize) and the last
hyperbatch's logits are computed with it (mx4_linear).  The graph, the teacher
and the labels are synthetic.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2601_01473_amd as ag  # noqa: E402
import synth  # noqa: E402


def teacher_of(off, idx, classes, k, gen):
    """Top logits of a planted teacher for every node: (logits [V, k], classes int32 [V, k], best class [V])."""
    V = len(off) - 1
    own = torch.randn(V, 16, device="cuda", generator=gen)
    deg = torch.from_numpy(np.diff(off)).cuda()
    src = torch.repeat_interleave(torch.arange(V, device="cuda"), deg)
    mean = ag.embedding_grad(own[torch.from_numpy(idx).cuda().long()], src, V) / deg.clamp(min=1).unsqueeze(1)
    z = (own + mean) @ torch.randn(16, classes, device="cuda", generator=gen)
    t, c = z.topk(k, dim=1)
    return t, c.int(), c[:, 0].int()


def mean_of_neighbours(batch):
    """The batch's targets and sampled edges as rows of its node list: (target rows [n], edge sources and targets
    [edges], the sources counted among the n targets, 1 / degree [n])."""
    rows, src, dst, inv, base, done = [], [], [], [], 0, 0
    for mb in batch.to_host(features=False):
        n, ptr, col = int(mb["layer_sizes"][0]), mb["row_ptr"][0], mb["col"][0]
        deg = np.diff(ptr)
        rows.append(base + np.arange(n))
        src.append(done + np.repeat(np.arange(n), deg))
        dst.append(base + col.astype(np.int64))
        inv.append(1.0 / np.maximum(deg, 1))
        base += len(mb["nodes"])
        done += n
    to = lambda x, t: torch.from_numpy(np.concatenate(x).astype(t)).cuda()  # noqa: E731
    return to(rows, np.int64), to(src, np.int64), to(dst, np.int64), to(inv, np.float32)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--scale", type=int, default=14, help="2^scale nodes")
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--classes", type=int, default=47)
    ap.add_argument("--top", type=int, default=8, help="teacher logits per node")
    ap.add_argument("--minibatches", type=int, default=8)
    ap.add_argument("--targets", type=int, default=256, help="per minibatch")
    ap.add_argument("--fanout", type=int, default=10)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--row-lr", type=float, default=0.25, help="rate of a node's row, per target that it takes part in")
    ap.add_argument("--head-lr", type=float, default=0.1)
    ap.add_argument("--seed", type=int, default=0)
    o = ap.parse_args(argv)

    gen = torch.Generator(device="cuda").manual_seed(o.seed)
    off, idx = synth.rmat_csr(o.scale, 16, seed=o.seed)
    V = len(off) - 1
    store = ag.Store(off, idx, synth.features(V, 4, seed=o.seed), 65536)
    t_logits, t_classes, labels = teacher_of(off, idx, o.classes, o.top, gen)
    labels[torch.rand(V, device="cuda", generator=gen) < 0.5] = -1          # half the nodes have no label

    table = torch.randn(V, o.dim, device="cuda", generator=gen)
    head = torch.randn(o.classes, o.dim, device="cuda", generator=gen) / o.dim ** 0.5
    n = o.minibatches * o.targets
    weight = torch.full((n,), 1.0 / n, device="cuda")
    losses, batch = [], None
    for step in range(o.steps):
        targets = synth.targets(V, n, seed=o.seed * 1000 + step)
        batch = store.prepare(targets.reshape(o.minibatches, o.targets), [o.fanout], seed=step, batch=batch)
        at, src, dst, inv = mean_of_neighbours(batch)
        node = torch.from_numpy(targets).cuda().long()

        h = batch.embedding(table, dtype=torch.bfloat16).float()
        x = (h[at] + ag.embedding_grad(h[dst] * inv[src].unsqueeze(1), src, n)).bfloat16()
        w16 = head.bfloat16()
        loss, dz = ag.distill_loss_grad(x @ w16.T, t_logits[node], t_classes[node], labels=labels[node],
                                        weight=weight, temperature=2.0, soft=0.7, hard=0.3)
        losses.append(loss.sum())

        dx = (dz @ w16).float()
        dh = ag.embedding_grad(torch.cat([dx, dx[src] * inv[src].unsqueeze(1)]), torch.cat([at, dst]), len(h))
        ids, rows, _ = batch.embedding_grad_rows(dh)        # as many rows as distinct nodes
        table.index_add_(0, ids, rows, alpha=-o.row_lr * n)
        head.add_((dz.T.contiguous() @ x).float(), alpha=-o.head_lr)

    losses = torch.stack(losses).tolist()
    z = x.float() @ head.T
    served = ag.mx4_linear(x, ag.mx4_quantize(head), dtype=torch.float32)
    best = t_classes[node][:, 0]
    result = dict(first_loss=losses[0], last_loss=losses[-1],
                  top1=float((z.argmax(1) == best).float().mean()),
                  top1_4bit=float((served.argmax(1) == best).float().mean()),
                  error_4bit=float((served - z).norm() / z.norm()))
    print("loss %.4f -> %.4f after %d hyperbatches; the teacher's first class on the last one: %.1f%%, in 4 bits %.1f%% "
          "(logits off by %.1f%%)" % (result["first_loss"], result["last_loss"], o.steps, 100 * result["top1"],
                                      100 * result["top1_4bit"], 100 * result["error_4bit"]))
    batch.close()
    store.close()
    return result


if __name__ == "__main__":
    main()
