"""A next-token model trained with the library's operators, its receivers kept in step by the transfer.

The trainer holds fp32 masters of an embedding, an RMS norm weight and a head, and takes AdamW steps on
synthetic text (every token has a few likely successors):

    embedding lookup -> [attention] -> RMS norm -> cross entropy of the head      (dte_embedding_*, dte_norm_*, dte_linear_ce_*)
    gradients -> [clipping] -> AdamW -> which BF16 elements changed                 (dte_extract_delta)
    scatter into the receivers' shards                                              (dte_apply)

With --heads there is a layer of causal attention with rotary positions in between (dte_rope, dte_attention_*), over
packed sequences of different lengths, two query heads to a key head; with --clip the global gradient norm is held
below a limit (dte_grad_sum_squares, dte_grad_clip).

Two receivers hold the embedding and the head cut over the vocabulary, the attention's projections cut over its heads,
in BF16.  With the same operators on their shards they score the next batch, and their loss is compared with the trainer's.

    python examples/train_and_sync.py [--steps 40] [--vocab 8192] [--hidden 512] [--tokens 4096] [--heads 0] [--clip 0]
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
HEAD_DIM = 64


def text(gen, successors, tokens):
    """`tokens` pairs (token, next token); the first eighth is a prompt, which carries no loss."""
    ids = torch.randint(0, successors.shape[0], (tokens,), generator=gen, device="cuda")
    pick = torch.randint(0, successors.shape[1], (tokens,), generator=gen, device="cuda")
    targets = successors[ids, pick]
    targets[:tokens // 8] = -100
    return ids, targets


def lengths_of(tokens):
    """Packed sequences of different lengths, down to one token."""
    out, left = [1], tokens - 1
    while left:
        out.append(min(left, 1 + 37 * len(out) % 301))
        left -= out[-1]
    return out


class Attention:
    """x = e + o(attention(rope(q(e)), rope(k(e)), v(e))) over the packed sequences of a batch: what the operators write, and
    the plan that the forward and the backward pass of every step share."""

    def __init__(self, tokens, heads, kv_heads):
        self.heads, self.kv_heads = heads, kv_heads
        lengths = lengths_of(tokens)
        self.starts = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()
        self.positions = torch.cat([torch.arange(n, device="cuda") for n in lengths])
        self.plan = torch.empty(dte.dte_attention_plan_bytes(tokens, len(lengths)), dtype=torch.uint8, device="cuda")
        dte.dte_attention_plan(self.starts, tokens, self.plan)
        self.frequencies = dte.dte_rope_frequencies(HEAD_DIM, 10000.0)[0].cuda()
        self.qkv, self.dqkv = (torch.empty(tokens, heads + 2 * kv_heads, HEAD_DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.a, self.da = (torch.empty(tokens, heads, HEAD_DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.lse = torch.empty(heads, tokens, device="cuda")
        self.workspace = torch.empty(dte.dte_attention_backward_workspace_bytes(tokens, heads), dtype=torch.uint8, device="cuda")

    def parts(self, t):
        return t[:, :self.heads], t[:, self.heads:-self.kv_heads], t[:, -self.kv_heads:]

    def forward(self, e, wqkv, wo):
        torch.matmul(e, wqkv.T, out=self.qkv.view(e.shape[0], -1))
        q, k, v = self.parts(self.qkv)
        dte.dte_rope(q, k, self.positions, self.frequencies)
        dte.dte_attention_forward(q, k, v, self.plan, self.a, self.lse)
        return self.a.flatten(1) @ wo.T

    def backward(self, dy, e, wqkv, wo):
        """(gradient of e, of wqkv and of wo) for a gradient dy of the output; the weights' in fp32."""
        torch.matmul(dy, wo, out=self.da.view(e.shape[0], -1))
        (q, k, v), (dq, dk, dv) = self.parts(self.qkv), self.parts(self.dqkv)
        dte.dte_attention_backward(q, k, v, self.a, self.lse, self.da, self.plan, dq, dk, dv, self.workspace)
        dte.dte_rope(dq, dk, self.positions, self.frequencies, inverse=True)
        d = self.dqkv.flatten(1)
        return d @ wqkv, d.float().T @ e.float(), dy.float().T @ self.a.flatten(1).float()


class Buffers:
    """What the operators write, and the workspace they share: allocated once."""

    def __init__(self, tokens, vocab, hidden, heads=0):
        self.e, self.h, self.dh, self.de = (torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda") for _ in range(4))
        self.rstd, self.lse, self.target_logit, self.loss = (torch.empty(tokens, device="cuda") for _ in range(4))
        size = max(dte.dte_linear_ce_forward_workspace_bytes(tokens, vocab, hidden),
                   dte.dte_linear_ce_backward_workspace_bytes(tokens, vocab, hidden),
                   dte.dte_norm_backward_workspace_bytes(tokens, hidden),
                   dte.dte_embedding_backward_workspace_bytes(tokens, hidden))
        self.workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.attention = Attention(tokens, heads, heads // 2) if heads else None


def train_step(b, embed, norm, head, ids, targets, grads, layer=()):
    """Loss of one batch and the gradients of the three weights, and of the attention layer's four (q, k, v, o), into grads (fp32)."""
    scale = math.sqrt(embed.shape[1])
    head16 = head.bfloat16()
    dte.dte_embedding_forward(embed, ids, b.e, scale=scale)
    x = b.e
    if layer:
        wqkv, wo = torch.cat(layer[:3]).bfloat16(), layer[3].bfloat16()
        x = b.e + b.attention.forward(b.e, wqkv, wo)
    dte.dte_norm_forward(x, norm, None, b.h, None, b.rstd, EPS, rms=True)
    dte.dte_linear_ce_forward(b.h, head16, targets, b.lse, None, b.loss, b.workspace)
    counted = (targets >= 0).sum()
    dloss = (targets >= 0) / counted.float()                     # mean over the tokens that count
    d_embed, d_norm, d_head = grads[:3]
    dte.dte_linear_ce_backward(b.h, head16, targets, b.lse, dloss, b.dh, d_head, b.workspace)
    dte.dte_norm_backward(b.dh, x, norm, None, b.rstd, b.de, d_norm, None, b.workspace, rms=True)
    if layer:
        de, dwqkv, dwo = b.attention.backward(b.de, b.e, wqkv, wo)
        for g, d in zip(grads[3:], (*dwqkv.split([w.shape[0] for w in layer[:3]]), dwo)):
            g.copy_(d)
        b.de += de
    dte.dte_embedding_backward(b.de, ids, d_embed, b.workspace, scale=scale)
    return b.loss.sum() / counted


def clip_gradients(grads, limit, total, workspace):
    """Global norm of the gradients below `limit`, in place."""
    dte.dte_grad_sum_squares(grads, total, workspace)
    dte.dte_grad_clip(grads, total, limit)


def receiver_loss(b, shards, vocab, hidden, ids, targets):
    """The same batch's loss from two receivers' BF16 shards: sums over receivers stand for the all-reduce."""
    rows, scale = vocab // 2, math.sqrt(hidden)
    part = torch.zeros_like(b.e, dtype=torch.float32)
    for r in range(2):
        out = torch.empty_like(part)
        dte.dte_embedding_forward(shards[r]["embed"].view(rows, hidden), ids, out, scale=scale, row_start=r * rows, vocab=vocab)
        part += out
    x = part.bfloat16()
    if b.attention:
        heads, kv_heads = b.attention.heads // 2, b.attention.kv_heads // 2
        own = Attention(ids.numel(), heads, kv_heads)            # a receiver's share of the heads
        x = x + sum(own.forward(x, shards[r]["qkv"].view(-1, hidden), shards[r]["o"].view(hidden, -1)).float() for r in range(2)).bfloat16()
    lse, logit = [], 0
    for r in range(2):
        dte.dte_norm_forward(x, shards[r]["norm"], None, b.h, None, None, EPS, rms=True)
        dte.dte_linear_ce_forward(b.h, shards[r]["head"].view(rows, hidden), targets, b.lse, b.target_logit, None, b.workspace,
                                  vocab_start=r * rows, vocab=vocab)
        lse.append(b.lse.clone())
        logit = logit + b.target_logit
    keep = targets >= 0
    return ((torch.logsumexp(torch.stack(lse), 0) - logit) * keep).sum() / keep.sum()


def run(steps=40, vocab=8192, hidden=512, tokens=4096, lr=2e-2, seed=0, say=print, heads=0, clip=0.0):
    # two query heads to a key head, and each of the two receivers holds key heads of its own
    if heads < 0 or heads % 4:
        raise ValueError("heads must be a multiple of 4 (0: no attention)")
    gen = torch.Generator("cuda").manual_seed(seed)
    successors = torch.randint(0, vocab, (vocab, 4), generator=gen, device="cuda")
    hp = dict(lr=lr, wd=0.01, eps=1e-8)
    names, shapes = ["embed", "norm", "head"], [(vocab, hidden), (hidden,), (vocab, hidden)]
    theta = [torch.empty(shapes[0], device="cuda").normal_(0, 0.02, generator=gen), torch.ones(hidden, device="cuda"),
             torch.empty(shapes[2], device="cuda").normal_(0, 0.02, generator=gen)]
    if heads:
        rows, kv_rows = heads * HEAD_DIM, heads // 2 * HEAD_DIM
        names += ["q", "k", "v", "o"]
        shapes += [(rows, hidden), (kv_rows, hidden), (kv_rows, hidden), (hidden, rows)]
        theta += [torch.empty(s, device="cuda").normal_(0, 0.02, generator=gen) for s in shapes[3:]]
    m, v = [torch.zeros_like(t) for t in theta], [torch.zeros_like(t) for t in theta]
    grads = [torch.empty_like(t) for t in theta]

    plan = Plan()
    src = [plan.add_tensor(n, s) for n, s in zip(names, shapes)]
    kinds = ["embed", "norm", "head"] + (["qkv", "o"] if heads else [])
    for r in range(2):
        plan.fused_rows("embed", [src[0]], r, 2)
        plan.replicated("norm", src[1], r)
        plan.fused_rows("head", [src[2]], r, 2)
        if heads:
            plan.fused_qkv("qkv", *src[3:6], r, 2, heads // 2, HEAD_DIM)
            plan.row_parallel("o", src[6], r, 2)
    layout = dte.Layout.from_plan(plan, 0)
    delta = layout.new_delta(layout.num_elements)

    def held(r):
        """What receiver r holds of the trainer's weights."""
        half = vocab // 2
        out = dict(embed=theta[0][r * half:(r + 1) * half], norm=theta[1], head=theta[2][r * half:(r + 1) * half])
        if heads:
            out["qkv"] = torch.cat([w.chunk(2)[r] for w in theta[3:6]])
            out["o"] = theta[6].chunk(2, 1)[r]
        return {k: t.bfloat16().reshape(-1) for k, t in out.items()}

    shards = [held(r) for r in range(2)]
    table = layout.shard_table([shards[r][k] for r in range(2) for k in kinds])

    b = Buffers(tokens, vocab, hidden, heads)
    total = torch.empty((), dtype=torch.float64, device="cuda")
    norm_space = torch.empty(dte.dte_grad_sum_squares_workspace_bytes(len(grads)), dtype=torch.uint8, device="cuda")
    losses, changed = [], 0
    for step in range(1, steps + 1):
        ids, targets = text(gen, successors, tokens)
        losses.append(float(train_step(b, *theta[:3], ids, targets, grads, theta[3:])))
        if clip:
            clip_gradients(grads, clip, total, norm_space)
        h = Hyper(step=step, **hp)
        for i in range(len(theta)):
            theta[i], m[i], v[i] = forward_adamw(theta[i], grads[i], m[i], v[i], h)
        dte.dte_extract_delta(layout, layout.source_tables(theta, m, v), *h.as_args(), delta)
        dte.dte_apply(layout, delta, table)
        changed = delta.total()
        if say and (step == 1 or step % 10 == 0):
            say(f"step {step:3d}  loss {losses[-1]:.4f}  {changed} of {layout.num_elements} BF16 elements changed")
    # the receivers against the trainer
    stale = sum(int((shards[r][k].view(torch.int16) != t.view(torch.int16)).sum()) for r in range(2) for k, t in held(r).items())
    ids, targets = text(gen, successors, tokens)
    here = float(train_step(b, theta[0].bfloat16(), theta[1].bfloat16(), theta[2], ids, targets, grads, theta[3:]))
    there = float(receiver_loss(b, shards, vocab, hidden, ids, targets))
    if say:
        say(f"next batch: trainer's loss {here:.5f}, receivers' {there:.5f}; {stale} of {layout.num_elements} shard elements differ "
            f"from the trainer's BF16 weights; least possible loss {math.log(4):.4f}")
    return dict(losses=losses, here=here, there=there, stale=stale, elements=layout.num_elements, changed=changed)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("steps", 40), ("vocab", 8192), ("hidden", 512), ("tokens", 4096)):
        ap.add_argument(f"--{name}", type=int, default=default)
    ap.add_argument("--heads", type=int, default=0, help="query heads of the attention layer, a multiple of 4 (0: no attention)")
    ap.add_argument("--clip", type=float, default=0.0)
    run(**vars(ap.parse_args()))
