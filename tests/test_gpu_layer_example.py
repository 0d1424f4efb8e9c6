"""The example's attention layer and clipping: the operators run together as a training step uses them, gradients against
automatic differentiation in 64 bits, the receivers' shards against the trainer's weights."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
try:
    import train_and_sync as example
finally:
    sys.path.pop(0)

pytestmark = pytest.mark.gpu


def model(theta, ids, targets, lengths, heads):
    """The example's model on 64-bit weights, with torch's operations and derivatives."""
    embed, norm, head, wq, wk, wv, wo = theta
    hidden, dim, group = embed.shape[1], example.HEAD_DIM, 2
    e = embed[ids] * math.sqrt(hidden)
    position = torch.cat([torch.arange(n, device="cuda") for n in lengths]).double()
    angle = torch.outer(position, 10000.0 ** (-torch.arange(dim // 2, device="cuda").double() * 2 / dim))[:, None]

    def turned(w, n):
        t = (e @ w.T).unflatten(1, (n, dim))
        a, b = t[..., :dim // 2], t[..., dim // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)

    q, k, v = turned(wq, heads), turned(wk, heads // group), (e @ wv.T).unflatten(1, (heads // group, dim))
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    out, at = [], 0
    for n in lengths:
        z = torch.einsum("ihd,jhd->hij", q[at:at + n], k[at:at + n]) / math.sqrt(dim)
        z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        out.append(torch.einsum("hij,jhd->ihd", z.softmax(-1), v[at:at + n]))
        at += n
    x = e + torch.cat(out).flatten(1) @ wo.T
    h = x * (x.square().mean(1, keepdim=True) + example.EPS).rsqrt() * norm
    return torch.nn.functional.cross_entropy(h @ head.T, targets, ignore_index=-100)


def test_gradients_of_the_whole_model():
    vocab, hidden, tokens, heads = 320, 128, 900, 4
    gen = torch.Generator("cuda").manual_seed(3)
    shapes = [(vocab, hidden), (hidden,), (vocab, hidden), (heads * 64, hidden), (heads * 32, hidden), (heads * 32, hidden), (hidden, heads * 64)]
    # weights that bf16 holds, so that both sides work on the same ones
    theta = [torch.empty(s, device="cuda").normal_(0, 0.08, generator=gen).bfloat16().float() for s in shapes]
    theta[1] += 1.0
    ids, targets = example.text(gen, torch.randint(0, vocab, (vocab, 4), generator=gen, device="cuda"), tokens)
    b = example.Buffers(tokens, vocab, hidden, heads)
    grads = [torch.empty_like(t) for t in theta]
    loss = example.train_step(b, *theta[:3], ids, targets, grads, theta[3:])
    leaves = [t.double().requires_grad_() for t in theta]
    want = model(leaves, ids, targets, example.lengths_of(tokens), heads)
    want.backward()
    # activations and their gradients are rounded to bf16 (2^-8 at most) at a dozen places between a weight and the loss and back
    room = 12 * 2.0 ** -8
    assert abs(float(loss) - float(want)) <= room * float(want)
    for g, leaf, name in zip(grads, leaves, ("embed", "norm", "head", "q", "k", "v", "o")):
        assert float((g.double() - leaf.grad).norm()) <= room * float(leaf.grad.norm()), name


def test_clipped_gradients_keep_their_direction():
    gen = torch.Generator("cuda").manual_seed(4)
    grads = [torch.empty(n, device="cuda").normal_(0, 1, generator=gen) for n in (5000, 7, 129)]
    before = [g.clone() for g in grads]
    import paper_2608_00455_b200 as dte

    total = torch.empty((), dtype=torch.float64, device="cuda")
    space = torch.empty(dte.dte_grad_sum_squares_workspace_bytes(3), dtype=torch.uint8, device="cuda")
    example.clip_gradients(grads, 2.0, total, space)
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in before))
    for g, w in zip(grads, before):
        # the norm, the factor and the product are rounded to fp32; its sums to 14 roundings
        assert bool(((g.double() - w.double() * (2.0 / norm)).abs() <= 10 * 2.0 ** -24 * w.double().abs()).all())


@pytest.mark.parametrize("heads,clip", [(4, 0.0), (4, 0.5), (0, 1.0)])
def test_training_with_attention_and_clipping_keeps_receivers_in_step(heads, clip):
    r = example.run(steps=4, vocab=512, hidden=128, tokens=1024, say=None, heads=heads, clip=clip)
    assert all(math.isfinite(x) for x in r["losses"])
    # an element the reconstruction takes for unchanged stays stale: the paper's method allows few of them
    assert r["stale"] <= r["elements"] * 1e-3
    # two receivers sum their heads' shares of the output: one more rounding to bf16 of x than the trainer's
    assert abs(r["here"] - r["there"]) <= 4 * 2.0 ** -8 * r["here"]
