"""A node classifier trained by the rewards of its own draws, its layers' inputs kept in 8 bits, then served with 8-bit weights.

    python examples/policy_nodes.py [--scale 14] [--dim 64] [--classes 47] [--steps 30]

A target's representation is its own row plus the mean of its sampled
neighbours' rows; a gated hidden layer and a linear head give its logits.  A
step is one hyperbatch:

    prepare, Batch.embedding    the targets' neighbourhoods and their rows
    policy_logprob      log-probabilities of the drawn classes, under the policy
                        that drew them and under the one that training began with
    mx8_quantize        the inputs of both layers, kept in 8 bits
    mx8_activation      the gated hidden layer, its input kept in 8 bits
    policy_loss_grad    the clipped loss of the draws' advantages with the
                        penalty for leaving the first policy, and its gradient
    mx8_weight_grad, mx8_activation_grad    the backward pass from what was kept

A draw's reward is 1 where it names the node's class; its advantage is the
reward less the mean over the target's draws.  After training both layers are
laid out in 8 bits once (int8_quantize), and the last hyperbatch's logits are
computed with them (int8_linear).  The graph and the classes are synthetic.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2601_01473_amd as ag  # noqa: E402
import synth  # noqa: E402
from examples.distill_nodes import mean_of_neighbours, teacher_of  # noqa: E402


def forward(x, w1, w2, keep=True):
    """(logits float32, hidden rows, kept hidden input)."""
    y, kept = ag.mx8_activation(x @ w1.bfloat16().T, "silu", gated=True, keep=keep)
    return (y @ w2.bfloat16().T).float(), y, kept


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--scale", type=int, default=14, help="2^scale nodes")
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--hidden", type=int, default=128)
    ap.add_argument("--classes", type=int, default=47)
    ap.add_argument("--minibatches", type=int, default=8)
    ap.add_argument("--targets", type=int, default=256, help="per minibatch")
    ap.add_argument("--draws", type=int, default=8, help="classes drawn per target")
    ap.add_argument("--updates", type=int, default=2, help="updates per hyperbatch")
    ap.add_argument("--fanout", type=int, default=10)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--lr", type=float, default=3.0)
    ap.add_argument("--kl", type=float, default=0.02)
    ap.add_argument("--seed", type=int, default=0)
    o = ap.parse_args(argv)

    gen = torch.Generator(device="cuda").manual_seed(o.seed)
    off, idx = synth.rmat_csr(o.scale, 16, seed=o.seed)
    V = len(off) - 1
    store = ag.Store(off, idx, synth.features(V, 4, seed=o.seed), 65536)
    _, _, labels = teacher_of(off, idx, o.classes, 1, gen)

    table = torch.randn(V, o.dim, device="cuda", generator=gen)
    w1 = torch.randn(2 * o.hidden, o.dim, device="cuda", generator=gen) / o.dim ** 0.5
    w2 = torch.randn(o.classes, o.hidden, device="cuda", generator=gen) / o.hidden ** 0.5
    first = w1.clone(), w2.clone()
    n, G = o.minibatches * o.targets, o.draws
    weight = torch.full((n * G,), 1.0 / (n * G), device="cuda")
    losses, rewards, batch = [], [], None
    for step in range(o.steps):
        targets = synth.targets(V, n, seed=o.seed * 1000 + step)
        batch = store.prepare(targets.reshape(o.minibatches, o.targets), [o.fanout], seed=step, batch=batch)
        at, src, dst, inv = mean_of_neighbours(batch)
        h = batch.embedding(table, dtype=torch.bfloat16).float()
        x = (h[at] + ag.embedding_grad(h[dst] * inv[src].unsqueeze(1), src, n)).bfloat16()
        kept_x = ag.mx8_quantize(x)

        z = forward(x, w1, w2, keep=False)[0]
        actions = torch.multinomial(torch.softmax(z, 1), G, replacement=True, generator=gen).view(-1)
        reward = (actions.view(n, G) == labels[torch.from_numpy(targets).cuda().long()].unsqueeze(1)).float()
        advantage = (reward - reward.mean(1, keepdim=True)).view(-1)
        old = ag.policy_logprob(z.repeat_interleave(G, 0), actions)
        ref = ag.policy_logprob(forward(x, *first, keep=False)[0].repeat_interleave(G, 0), actions)
        rewards.append(reward.mean())

        for _ in range(o.updates):
            z, y, kept_h = forward(x, w1, w2)
            kept_y = ag.mx8_quantize(y)
            loss, _, dz = ag.policy_loss_grad(z.repeat_interleave(G, 0), actions, advantage, old, ref_logp=ref,
                                              weight=weight, kl=o.kl)
            dz = dz.view(n, G, o.classes).sum(1)
            dy = dz.bfloat16() @ w2.bfloat16()
            dw2 = ag.mx8_weight_grad(dz, kept_y)
            dw1 = ag.mx8_weight_grad(ag.mx8_activation_grad(dy, kept_h, "silu", gated=True), kept_x, dtype=torch.float32)
            w2.add_(dw2, alpha=-o.lr)
            w1.add_(dw1, alpha=-o.lr)
        losses.append(loss.sum())

    z = forward(x, w1, w2, keep=False)[0]
    # served: both layers' weights in 8 bits, their rows quantised on the way in
    y, _ = ag.mx8_activation(ag.int8_linear(x, ag.int8_quantize(w1)), "silu", gated=True, keep=False)
    served = ag.int8_linear(y, ag.int8_quantize(w2), dtype=torch.float32)
    result = dict(loss=float(losses[-1]), first_reward=float(rewards[0]), last_reward=float(rewards[-1]),
                  error_8bit=float((served - z).norm() / z.norm()),
                  same_class=float((served.argmax(1) == z.argmax(1)).float().mean()))
    print("mean reward %.4f -> %.4f after %d hyperbatches; served in 8 bits: logits off by %.2f%%, the same class for %.1f%%"
          % (result["first_reward"], result["last_reward"], o.steps, 100 * result["error_8bit"], 100 * result["same_class"]))
    batch.close()
    store.close()
    return result


if __name__ == "__main__":
    main()
