"""A next-token model trained with the library's operators, its receivers kept in step by the transfer.

The trainer holds fp32 masters of an embedding, an RMS norm weight and a head, and takes AdamW steps on
synthetic text (every token has a few likely successors):

    embedding lookup -> RMS norm -> cross entropy of the head      (dte_embedding_*, dte_norm_*, dte_linear_ce_*)
    gradients -> AdamW -> which BF16 elements changed               (dte_extract_delta)
    scatter into the receivers' shards                              (dte_apply)

Two receivers hold the embedding and the head cut over the vocabulary, in BF16.  With the same operators on their
shards they score the next batch, and their loss is compared with the trainer's.

    python examples/train_and_sync.py [--steps 40] [--vocab 8192] [--hidden 512] [--tokens 4096]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_00455_b200 as dte                                        # noqa: E402
from synth.plans import Plan                                               # noqa: E402
from synth.tensors import Hyper, forward_adamw                             # noqa: E402

EPS = 1e-6


def text(gen, successors, tokens):
    """`tokens` pairs (token, next token); the first eighth is a prompt, which carries no loss."""
    ids = torch.randint(0, successors.shape[0], (tokens,), generator=gen, device="cuda")
    pick = torch.randint(0, successors.shape[1], (tokens,), generator=gen, device="cuda")
    targets = successors[ids, pick]
    targets[:tokens // 8] = -100
    return ids, targets


class Buffers:
    """What the operators write, and the workspace they share: allocated once."""

    def __init__(self, tokens, vocab, hidden):
        self.e, self.h, self.dh, self.de = (torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda") for _ in range(4))
        self.rstd, self.lse, self.target_logit, self.loss = (torch.empty(tokens, device="cuda") for _ in range(4))
        size = max(dte.dte_linear_ce_forward_workspace_bytes(tokens, vocab, hidden),
                   dte.dte_linear_ce_backward_workspace_bytes(tokens, vocab, hidden),
                   dte.dte_norm_backward_workspace_bytes(tokens, hidden),
                   dte.dte_embedding_backward_workspace_bytes(tokens, hidden))
        self.workspace = torch.empty(size, dtype=torch.uint8, device="cuda")


def train_step(b, embed, norm, head, ids, targets, grads):
    """Loss of one batch and the gradients of the three weights, into grads (fp32)."""
    scale = math.sqrt(embed.shape[1])
    head16 = head.bfloat16()
    dte.dte_embedding_forward(embed, ids, b.e, scale=scale)
    dte.dte_norm_forward(b.e, norm, None, b.h, None, b.rstd, EPS, rms=True)
    dte.dte_linear_ce_forward(b.h, head16, targets, b.lse, None, b.loss, b.workspace)
    counted = (targets >= 0).sum()
    dloss = (targets >= 0) / counted.float()                     # mean over the tokens that count
    d_embed, d_norm, d_head = grads
    dte.dte_linear_ce_backward(b.h, head16, targets, b.lse, dloss, b.dh, d_head, b.workspace)
    dte.dte_norm_backward(b.dh, b.e, norm, None, b.rstd, b.de, d_norm, None, b.workspace, rms=True)
    dte.dte_embedding_backward(b.de, ids, d_embed, b.workspace, scale=scale)
    return b.loss.sum() / counted


def receiver_loss(b, shards, vocab, hidden, ids, targets):
    """The same batch's loss from two receivers' BF16 shards: sums over receivers stand for the all-reduce."""
    rows, scale = vocab // 2, math.sqrt(hidden)
    part = torch.zeros_like(b.e, dtype=torch.float32)
    for r in range(2):
        out = torch.empty_like(part)
        dte.dte_embedding_forward(shards[r]["embed"].view(rows, hidden), ids, out, scale=scale, row_start=r * rows, vocab=vocab)
        part += out
    x = part.bfloat16()
    lse, logit = [], 0
    for r in range(2):
        dte.dte_norm_forward(x, shards[r]["norm"], None, b.h, None, None, EPS, rms=True)
        dte.dte_linear_ce_forward(b.h, shards[r]["head"].view(rows, hidden), targets, b.lse, b.target_logit, None, b.workspace,
                                  vocab_start=r * rows, vocab=vocab)
        lse.append(b.lse.clone())
        logit = logit + b.target_logit
    keep = targets >= 0
    return ((torch.logsumexp(torch.stack(lse), 0) - logit) * keep).sum() / keep.sum()


def run(steps=40, vocab=8192, hidden=512, tokens=4096, lr=2e-2, seed=0, say=print):
    gen = torch.Generator("cuda").manual_seed(seed)
    successors = torch.randint(0, vocab, (vocab, 4), generator=gen, device="cuda")
    hp = dict(lr=lr, wd=0.01, eps=1e-8)
    shapes = [(vocab, hidden), (hidden,), (vocab, hidden)]       # embedding, norm, head
    theta = [torch.empty(shapes[0], device="cuda").normal_(0, 0.02, generator=gen), torch.ones(hidden, device="cuda"),
             torch.empty(shapes[2], device="cuda").normal_(0, 0.02, generator=gen)]
    m, v = [torch.zeros_like(t) for t in theta], [torch.zeros_like(t) for t in theta]
    grads = [torch.empty_like(t) for t in theta]

    plan = Plan()
    src = [plan.add_tensor("embed", shapes[0]), plan.add_tensor("norm", shapes[1]), plan.add_tensor("head", shapes[2])]
    for r in range(2):
        plan.fused_rows("embed", [src[0]], r, 2)
        plan.replicated("norm", src[1], r)
        plan.fused_rows("head", [src[2]], r, 2)
    layout = dte.Layout.from_plan(plan, 0)
    delta = layout.new_delta(layout.num_elements)
    half = vocab // 2
    shards = [dict(embed=theta[0][r * half:(r + 1) * half].bfloat16().reshape(-1), norm=theta[1].bfloat16(),
                   head=theta[2][r * half:(r + 1) * half].bfloat16().reshape(-1)) for r in range(2)]
    table = layout.shard_table([shards[r][k] for r in range(2) for k in ("embed", "norm", "head")])

    b = Buffers(tokens, vocab, hidden)
    losses, changed = [], 0
    for step in range(1, steps + 1):
        ids, targets = text(gen, successors, tokens)
        losses.append(float(train_step(b, *theta, ids, targets, grads)))
        h = Hyper(step=step, **hp)
        for i in range(3):
            theta[i], m[i], v[i] = forward_adamw(theta[i], grads[i], m[i], v[i], h)
        dte.dte_extract_delta(layout, layout.source_tables(theta, m, v), *h.as_args(), delta)
        dte.dte_apply(layout, delta, table)
        changed = delta.total()
        if say and (step == 1 or step % 10 == 0):
            say(f"step {step:3d}  loss {losses[-1]:.4f}  {changed} of {layout.num_elements} BF16 elements changed")
    # the receivers against the trainer
    stale = 0
    for r in range(2):
        want = [theta[0][r * half:(r + 1) * half], theta[1], theta[2][r * half:(r + 1) * half]]
        for k, t in zip(("embed", "norm", "head"), want):
            stale += int((shards[r][k].view(torch.int16) != t.bfloat16().reshape(-1).view(torch.int16)).sum())
    ids, targets = text(gen, successors, tokens)
    here = float(train_step(b, theta[0].bfloat16(), theta[1].bfloat16(), theta[2], ids, targets, grads))
    there = float(receiver_loss(b, shards, vocab, hidden, ids, targets))
    if say:
        say(f"next batch: trainer's loss {here:.5f}, receivers' {there:.5f}; {stale} of {layout.num_elements} shard elements differ "
            f"from the trainer's BF16 weights; least possible loss {math.log(4):.4f}")
    return dict(losses=losses, here=here, there=there, stale=stale, elements=layout.num_elements, changed=changed)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("steps", 40), ("vocab", 8192), ("hidden", 512), ("tokens", 4096)):
        ap.add_argument(f"--{name}", type=int, default=default)
    run(**vars(ap.parse_args()))
