"""Policy training with an every-iteration snapshot, all of it on the device.

A small policy (one projection and a vocabulary head over fixed features) learns to prefer some
tokens.  An iteration is: logits by two matrix products; the clipped policy loss with its gradient,
written over the logits; the weights' gradients by three more products; the norm of all gradients; and
the clipped AdamW step that writes the new state into one of two alternating snapshots.  No value
comes back to the host in between: an fp16 overflow leaves the update out by itself, and is seen in the
statistics when they are looked at.  In the end a newcomer takes the last snapshot over: verified, loaded,
and compared.

    python examples/policy_training.py [--steps 30] [--half bf16|fp16]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2512_03644_amd import binding as ff  # noqa: E402

DEV = "cuda:0"
TOKENS, FEATURES, HIDDEN, VOCAB = 512, 192, 256, 4099
CLIP, BETA, MAX_NORM = 0.2, 0.02, 0.05


class Policy:
    """16-bit working weights with fp32 master weights and moments, and the plan over all of them."""

    def __init__(self, half, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        shapes = [(HIDDEN, FEATURES), (VOCAB, HIDDEN)]
        self.master = [torch.randn(s, generator=g, device=DEV) / s[1] ** 0.5 for s in shapes]
        self.w16 = [p.to(half) for p in self.master]
        self.m = [torch.zeros_like(p) for p in self.master]
        self.v = [torch.zeros_like(p) for p in self.master]
        self.tensors = [t.view(-1) for group in zip(self.w16, self.master, self.m, self.v) for t in group]
        kinds = [ff.FF_KIND_W16, ff.FF_KIND_MASTER, ff.FF_KIND_M, ff.FF_KIND_V] * len(shapes)
        self.plan = ff.ff_snapshot_plan(self.tensors, 1 << 16, 0, kinds, [k // 4 for k in range(len(kinds))])


def train(steps=30, half=torch.bfloat16, seed=0, report=print):
    """Returns (losses, norms, weights and newcomer's weights) after `steps` iterations."""
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    features = torch.randn(TOKENS, FEATURES, generator=g, device=DEV).to(half)
    targets = torch.randint(0, VOCAB, (TOKENS,), generator=g, device=DEV)
    # even tokens were good, odd ones bad; every eighth position is a prompt's and counts nothing
    advantages = torch.where(targets % 2 == 0, 1.0, -1.0)
    weights = torch.full((TOKENS,), 1.0 / (TOKENS - TOKENS // 8), device=DEV)
    weights[::8] = 0.0

    policy = Policy(half, seed)
    loss_scale = 1024.0 if half == torch.float16 else 1.0
    hp = dict(lr=2e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.01)

    # what a program makes once: the list of gradients, statistics, workspaces, two snapshots
    grads = [torch.zeros_like(w) for w in policy.w16]
    flat = [x.view(-1) for x in grads]
    grad_list = ff.ff_grad_list(flat)
    stats, norm_space = ff.GradStats(DEV), ff.alloc_grad_workspace(grad_list, DEV)
    loss_stats, loss_space = ff.PolicyStats(DEV), ff.alloc_policy_workspace(TOKENS, VOCAB, DEV)
    logp, token_loss = torch.empty(TOKENS, device=DEV), torch.empty(TOKENS, device=DEV)
    snapshots = [ff.alloc_outputs(policy.plan, DEV) for _ in range(2)]
    ff.ff_pack(policy.plan, snapshots[0][0], snapshots[0][1])

    def forward():
        hidden = features @ policy.w16[0].t()
        return hidden, hidden @ policy.w16[1].t()

    # the policy that made the tokens, which is the reference as well
    _, logits = forward()
    old_logp = torch.empty(TOKENS, device=DEV)
    zeros, ones = torch.zeros(TOKENS, device=DEV), torch.ones(TOKENS, device=DEV)
    scored = ff.policy_batch(logits, targets, zeros, zeros, ones)
    ff.ff_policy_loss(scored, old_logp, token_loss, loss_stats, loss_space)

    losses, norms = [], []
    for step in range(1, steps + 1):  # (iterations: one whose update is left out counts in the bias correction)
        hidden, logits = forward()
        batch = ff.policy_batch(logits, targets, old_logp, advantages, weights, old_logp, CLIP, CLIP, BETA, loss_scale)
        ff.ff_policy_loss(batch, logp, token_loss, loss_stats, loss_space, dlogits=logits)
        torch.mm(logits.t(), hidden, out=grads[1])
        torch.mm((logits @ policy.w16[1]).t(), features, out=grads[0])
        ff.ff_grad_norm(grad_list, stats, norm_space, MAX_NORM, 1.0 / loss_scale)
        old, new = snapshots[(step - 1) % 2], snapshots[step % 2]
        ff.ff_adam_step_clipped(policy.plan, flat, dict(hp, step=step), stats, new[0], new[1], old[0])
        losses.append(loss_stats.loss.clone())
        norms.append(stats.norm.clone())
    losses, norms = [float(x) for x in losses], [float(x) for x in norms]
    report("loss %.4f -> %.4f, gradient norm %.3f -> %.3f (clipped to %.2f), %d of %d tokens clipped in the last iteration"
           % (losses[0], losses[-1], norms[0], norms[-1], MAX_NORM, int(loss_stats.n_clipped), int(loss_stats.n_tokens)))

    # failover: a newcomer of the same layout checks and loads what the last step has written
    newcomer = Policy(half, seed + 99)
    chunks, crcs, bad, n_bad = snapshots[steps % 2]
    ff.ff_restore_checked(newcomer.plan, policy.plan.layout_id, chunks, crcs, bad, n_bad)
    report("%d bytes in %d chunks, %d damaged" % (policy.plan.payload_bytes, policy.plan.num_chunks, int(n_bad)))
    if int(n_bad):
        raise RuntimeError("the snapshot is damaged")
    return losses, norms, policy.w16, newcomer.w16


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--half", choices=("bf16", "fp16"), default="bf16")
    a = ap.parse_args()
    _, _, trained, taken_over = train(a.steps, torch.bfloat16 if a.half == "bf16" else torch.float16)
    same = all(torch.equal(x, y) for x, y in zip(trained, taken_over))
    print("the newcomer's weights are the trained ones" if same else "the newcomer's weights differ")
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
