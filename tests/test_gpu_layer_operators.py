"""The operators inside and behind the model's layers - rotary positions, causal attention over packed sequences, the
global gradient norm with clipping - element by element against their formulas in 64 bits, at the sizes, strides, masks and
types where they can go wrong; gradients against differences as well.

Every tolerance is an element-wise bound made from the operator's own rounding steps: U is the rounding of the output
type, E = 2^-24 one fp32 rounding.  The tensor cores truncate: a sum of n products is off by at most n units of
2^-23 of the sum of magnitudes.
"""
import math

import pytest
import torch

import paper_2608_00455_b200 as dte

pytestmark = pytest.mark.gpu

F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
E = 2.0 ** -24
DEV = "cuda"


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def normal(seed, shape, std=1.0, dtype=F32, mean=0.0):
    return torch.empty(shape, dtype=F32, device=DEV).normal_(mean, std, generator=gen(seed)).to(dtype)


def assert_within(got, want, bound, what):
    got = got.to(F64)
    assert got.shape == want.shape, what
    bad = ~((got - want).abs() <= bound)
    if bool(bad.any()):
        i = int(bad.reshape(-1).nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: got {got.reshape(-1)[i].item()!r}, "
                             f"want {want.reshape(-1)[i].item()!r} +- {bound.expand_as(want).reshape(-1)[i].item():.3g}")


def workspace(nbytes):
    # filled with NaN patterns: nothing may depend on what a workspace holds
    return torch.full((max(16, nbytes),), 0xFF, dtype=torch.uint8, device=DEV)


def same_bits(a, b):
    if a.dtype == BF16:
        return torch.equal(a.view(torch.int16), b.view(torch.int16))
    return torch.equal(a.view(torch.int32), b.view(torch.int32))


# ---- rotary positions -----------------------------------------------------------------------------------------

def heads_of(seed, tokens, heads, dim, dtype, extra=0, offset=0):
    """tokens x heads x dim, a token's heads side by side, rows heads * dim + extra apart, `offset` elements into an allocation."""
    ld = heads * dim + extra
    buf = normal(seed, (offset + max(1, tokens) * ld,), 1.0, dtype)
    return buf[offset:offset + tokens * ld].view(tokens, ld)[:, :heads * dim].unflatten(1, (heads, dim))


def rope_want(x, pos, freq, interleaved, amplitude, inverse):
    """(result, bound) in 64 bits."""
    rot = 2 * freq.numel()
    keep = (pos >= 0)[:, None, None]
    angle = pos.to(F64)[:, None] * freq
    amp = torch.tensor(amplitude, dtype=F32).to(F64).item()
    c, s = angle.cos()[:, None] * amp, angle.sin()[:, None] * amp * (-1 if inverse else 1)
    x = x.to(F64)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    lo, hi = a * c - b * s, b * c + a * s
    # the angle: two 64-bit roundings of the product, once more in the oracle's, and 2^-28 of a turn; sine and cosine 2 units, the
    # amplitude's product; then three fp32 roundings
    off = ((angle.abs() * 2.0 ** -51 + 2 * math.pi * 2.0 ** -28 + 4 * E)[:, None] * amp + 3 * E * amp) * (a.abs() + b.abs())
    want, bound = x.clone(), torch.zeros_like(x)
    ends = [(slice(0, rot, 2), slice(1, rot, 2))] if interleaved else [(slice(0, rot // 2), slice(rot // 2, rot))]
    for l, h in ends:
        want[..., l], want[..., h] = torch.where(keep, lo, a), torch.where(keep, hi, b)
        bound[..., l], bound[..., h] = torch.where(keep, off, 0.0), torch.where(keep, off, 0.0)
    return want, bound


@pytest.mark.parametrize("dim,rot", [(2, 2), (8, 8), (9, 6), (16, 16), (64, 32), (66, 66), (80, 40), (128, 128), (128, 64), (128, 2), (256, 64), (1024, 1024)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rope(dim, rot, interleaved, dtype):
    freq = (10000.0 ** (-torch.arange(rot // 2, dtype=F64) * 2 / rot)).to(DEV)
    for tokens, hq, hk, extra, offset, inverse, ids in ((1, 1, 1, 0, 0, False, torch.int64), (5, 3, 2, 8, 8, True, torch.int32),
                                                       (37, 4, 1, 3, 1, False, torch.int32), (6, 2, 0, 2, 2, True, torch.int64)):
        q = heads_of(1, tokens, hq, dim, dtype, extra, offset)
        k = heads_of(2, tokens, hk, dim, dtype, extra, offset) if hk else None
        pos = torch.randint(0, 200000, (tokens,), generator=gen(3), device=DEV, dtype=ids)
        pos[0] = 2 ** 31 - 1
        if tokens > 3:
            pos[1], pos[2] = 0, -1
        for side in (q, k):
            if side is not None and tokens > 4 and rot < dim:
                side[3, :, rot:] = float("nan")                    # copied columns may hold anything
        outs = [None if t is None else heads_of(4, tokens, t.shape[1], dim, dtype, extra, offset) for t in (q, k)]
        dte.dte_rope(q, k, pos, freq, outs[0], outs[1], interleaved=interleaved, amplitude=1.25, inverse=inverse)
        want = [None if t is None else rope_want(t, pos, freq, interleaved, 1.25, inverse) for t in (q, k)]
        for t, o, w in zip((q, k), outs, want):
            if t is None:
                continue
            assert same_bits(o[..., rot:], t[..., rot:].contiguous())
            assert_within(o[..., :rot], w[0][..., :rot], w[1][..., :rot] + U[dtype] * w[0][..., :rot].abs() * 1.01 + 1e-38, f"{tokens}")
            if tokens > 3:
                assert same_bits(o[2], t[2].contiguous())
        dte.dte_rope(q, k, pos, freq, interleaved=interleaved, amplitude=1.25, inverse=inverse)      # in place: the same bits
        for t, o in zip((q, k), outs):
            assert t is None or same_bits(t.contiguous(), o.contiguous())


def test_rope_at_position_zero_and_its_inverse():
    freq, amplitude = dte.dte_rope_frequencies(64, 1e6)
    assert amplitude == 1.0
    freq = freq.to(DEV)
    q, zero = normal(5, (9, 2, 64)), torch.zeros(9, dtype=torch.int64, device=DEV)
    out = torch.empty_like(q)
    dte.dte_rope(q, None, zero, freq, out)
    assert torch.equal(out, q)
    pos = torch.arange(9, device=DEV) * 1234567
    d = normal(6, (9, 2, 64))
    back = torch.empty_like(d)
    dte.dte_rope(q, None, pos, freq, out, interleaved=True, amplitude=1.5)
    dte.dte_rope(d, None, pos, freq, back, interleaved=True, amplitude=1.5, inverse=True)
    # adjoint: <R q, d> = <q, R^T d>
    a, b = (out.to(F64) * d.to(F64)).sum(), (q.to(F64) * back.to(F64)).sum()
    assert abs(float(a - b)) <= 40 * E * float((out.to(F64) * d.to(F64)).abs().sum())


def test_rope_shapes_that_hold_nothing():
    freq = torch.ones(4, dtype=F64, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    dte.dte_rope(torch.empty(0, 3, 8, device=DEV), torch.empty(0, 1, 8, device=DEV), none, freq)


# ---- attention ------------------------------------------------------------------------------------------------

def starts_of(lengths, front=0, dtype=torch.int32):
    s = [front]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=dtype, device=DEV)


def plan_of(starts, tokens, flags=None):
    plan = workspace(dte.dte_attention_plan_bytes(tokens, starts.numel() - 1))
    dte.dte_attention_plan(starts, tokens, plan, flags)
    return plan


class Batch:
    """Inputs of an attention call: rows of no sequence hold NaN, outputs a value that must stay there."""

    def __init__(self, lengths, hq, hk, dim, front=0, behind=0, fused=False, seed=1, std=1.0, ids=torch.int32, scale=None):
        self.lengths, self.hq, self.hk, self.dim, self.front = lengths, hq, hk, dim, front
        self.group, self.scale = hq // hk, dim ** -0.5 if scale is None else scale
        self.tokens = front + sum(lengths) + behind
        if fused:
            x = normal(seed, (self.tokens, hq + 2 * hk + 1, dim), std, BF16)
            self.q, self.k, self.v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:hq + 2 * hk]
        else:
            self.q, self.k, self.v = (normal(seed + i, (self.tokens, h, dim), std, BF16) for i, h in enumerate((hq, hk, hk)))
        self.dout = normal(seed + 7, (self.tokens, hq, dim), 1.0, BF16)
        self.member = torch.zeros(self.tokens, dtype=torch.bool, device=DEV)
        self.member[front:front + sum(lengths)] = True
        for t in (self.q, self.k, self.v, self.dout):
            t[~self.member] = float("nan")
        self.starts = starts_of(lengths, front, ids)
        self.plan = plan_of(self.starts, self.tokens)
        self.out = torch.full((self.tokens, hq, dim), 3.0, dtype=BF16, device=DEV)
        self.lse = torch.full((hq, self.tokens), 3.0, device=DEV)
        self.grads = [torch.full((self.tokens, h, dim), 3.0, dtype=BF16, device=DEV) for h in (hq, hk, hk)]

    def forward(self, stream=None):
        dte.dte_attention_forward(self.q, self.k, self.v, self.plan, self.out, self.lse, scale=self.scale, stream=stream)

    def backward(self, stream=None, ws=None):
        if ws is None:
            ws = workspace(dte.dte_attention_backward_workspace_bytes(self.tokens, self.hq))
        dte.dte_attention_backward(self.q, self.k, self.v, self.out, self.lse, self.dout, self.plan, *self.grads, ws, scale=self.scale,
                                   stream=stream)

    def pieces(self):
        a = self.front
        for n in self.lengths:
            for h in range(self.hq):
                if n:
                    yield slice(a, a + n), h, h // self.group
            a += n

    def scores(self, rows, h, kh):
        q, k = self.q[rows, h].to(F64), self.k[rows, kh].to(F64)
        n = q.shape[0]
        seen = torch.ones(n, n, dtype=torch.bool, device=DEV).tril_()
        z = (q @ k.T) * self.scale
        # one unit per product, two fp32 roundings of the scaling
        off = (q.abs() @ k.abs().T) * self.scale * (self.dim * 2 * E) + 3 * E * z.abs()
        return z.masked_fill(~seen, -math.inf), off.masked_fill(~seen, 0.0), q, k, seen

    def check_forward(self):
        for rows, h, kh in self.pieces():
            z, off, _, _, seen = self.scores(rows, h, kh)
            lse = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[:, None])
            # exponentials: 2^-22, and the roundings of their arguments, which stay below |z - lse| + 8 in base e
            rel = off.amax(1, keepdim=True) * 2 + E * (8 + 4 * (z - lse[:, None]).masked_fill(~seen, 0.0).abs() + 4 * lse[:, None].abs())
            v = self.v[rows, kh].to(F64)
            n = v.shape[0]
            want = p @ v
            bound = (p * (rel + U[BF16] * 1.01 + n * 2 * E)) @ v.abs() + U[BF16] * 1.01 * want.abs() + 1e-30
            assert_within(self.out[rows, h], want, bound, f"out {rows} {h}")
            slack = off.amax(1) + (p * rel).sum(1) + n * E + 4 * E * (1 + lse.abs() + z.masked_fill(~seen, 0.0).abs().amax(1))
            assert_within(self.lse[h, rows], lse, slack, f"lse {rows} {h}")
        assert bool((self.out[~self.member] == 3.0).all()) and bool((self.lse[:, ~self.member] == 3.0).all())

    def check_backward(self):
        """Against the documented formulas, from the outputs that were passed."""
        want = [torch.zeros(g.shape, dtype=F64, device=DEV) for g in self.grads]
        bound = [torch.zeros(g.shape, dtype=F64, device=DEV) for g in self.grads]
        for rows, h, kh in self.pieces():
            z, off, q, k, seen = self.scores(rows, h, kh)
            lse = self.lse[h, rows].to(F64)[:, None]
            p = torch.exp(z - lse)
            rel = off + E * (8 + 4 * (z - lse).masked_fill(~seen, 0.0).abs() + 4 * lse.abs())
            v, do, o = self.v[rows, kh].to(F64), self.dout[rows, h].to(F64), self.out[rows, h].to(F64)
            n, d = v.shape
            dp, delta = do @ v.T, (do * o).sum(1, keepdim=True)
            dz = p * (dp - delta)
            dz[0] = 0.0                                    # one key: the weight is constant
            dp_off = d * 2 * E * (do.abs() @ v.abs().T + (do * o).abs().sum(1, keepdim=True))
            dz_off = p * (rel * (dp.abs() + delta.abs()) + dp_off) + U[BF16] * 1.01 * dz.abs()
            dz_off[0] = 0.0
            long = n * 2 * E
            want[0][rows, h] = self.scale * dz @ k
            bound[0][rows, h] = self.scale * (dz_off + long * dz.abs()) @ k.abs()
            want[1][rows, kh] += self.scale * dz.T @ q
            bound[1][rows, kh] += self.scale * (dz_off + self.group * long * dz.abs()).T @ q.abs()
            want[2][rows, kh] += p.T @ do
            bound[2][rows, kh] += (p * (rel + U[BF16] * 1.01 + self.group * long)).T @ do.abs()
        for g, w, b, name in zip(self.grads, want, bound, ("dq", "dk", "dv")):
            assert_within(g[self.member], w[self.member], (b + U[BF16] * 1.01 * w.abs() + 4 * E * w.abs() + 1e-30)[self.member], name)
            assert bool((g[~self.member] == 3.0).all()), name


LENGTHS = [[1], [1, 1, 1], [2, 0, 3], [63], [64, 65], [127], [128], [129], [0, 0, 255, 256, 257, 0], [384, 1, 130], [700], [5] * 40, [1025]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: "-".join(map(str, v[:6])))
@pytest.mark.parametrize("hq,hk,dim", [(2, 1, 128), (1, 1, 128), (3, 1, 64), (4, 4, 64)])
def test_attention_lengths(lengths, hq, hk, dim):
    b = Batch(lengths, hq, hk, dim, front=3, behind=5, fused=True)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("dim", [8, 16, 24, 40, 56, 72, 80, 96, 104, 120])
@pytest.mark.parametrize("hq,hk,fused", [(2, 2, False), (8, 2, True), (5, 1, False), (6, 2, True)])
def test_attention_heads_and_widths(dim, hq, hk, fused):
    b = Batch([150, 31, 300], hq, hk, dim, behind=2, fused=fused, ids=torch.int64)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


# Few key tiles of many query heads: the heads of a key head are cut into parts, whose sums are added up.
@pytest.mark.parametrize("lengths,hq,hk,dim", [([300], 8, 1, 128), ([129], 64, 1, 72), ([700, 20], 24, 2, 64), ([512], 32, 4, 40), ([1025, 0, 3, 1], 16, 1, 104),
                                               ([900], 12, 1, 128), ([128, 128], 32, 1, 96), ([2050], 32, 1, 128)])
def test_attention_of_few_sequences_and_many_heads(lengths, hq, hk, dim):
    b = Batch(lengths, hq, hk, dim, front=1, behind=130, fused=True)
    b.forward()
    b.backward()
    b.check_backward()
    first = [t.clone() for t in b.grads]
    ws = workspace(dte.dte_attention_backward_workspace_bytes(b.tokens, b.hq))
    for _ in range(3):                                     # whichever part comes last, with what an earlier call left
        b.backward(None, ws)
        for t, w in zip(b.grads, first):
            assert same_bits(t, w)


def test_attention_replayed_where_heads_are_cut_and_where_not():
    long, short = Batch([640, 0, 0, 0], 16, 1, 64), Batch([160] * 4, 16, 1, 64, seed=50)
    work = Batch([640, 0, 0, 0], 16, 1, 64, seed=70)
    ws = workspace(dte.dte_attention_backward_workspace_bytes(640, 16))

    def step():
        dte.dte_attention_plan(work.starts, 640, work.plan)
        work.forward()
        work.backward(None, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for other in (long, short, long):
        work.starts.copy_(other.starts)
        for name in ("q", "k", "v", "dout"):
            getattr(work, name).copy_(getattr(other, name))
        graph.replay()
        other.forward()
        other.backward()
        for t, w in zip(work.grads, other.grads):
            assert same_bits(t, w)
        other.check_backward()


@pytest.mark.parametrize("std,scale", [(6.0, None), (1.0, 3.0), (0.05, None), (1.0, 1e-3), (3.0, 0.7)])
def test_attention_of_peaked_and_flat_scores(std, scale):
    b = Batch([300, 140], 4, 2, 128, std=std, scale=scale)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


def test_attention_scores_that_grow_along_the_keys():
    # the running maximum moves in every tile, by little and by much
    for step in (0.01, 0.3, 5.0):
        b = Batch([900], 2, 1, 64, std=0.1)
        b.k[:, 0, 0] = (torch.arange(900, device=DEV) * step).to(BF16)
        b.q[:, :, 0] = 2.0
        b.forward()
        b.check_forward()
        b.backward()
        b.check_backward()


def test_attention_of_long_sequences():
    b = Batch([2600, 4200], 2, 1, 128, behind=3)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


def test_attention_where_scores_are_infinite():
    # keys that no query can choose: their scores are -inf; a whole first tile of them, too
    for blocked in (slice(3, 9), slice(0, 128), slice(0, 200)):
        b = Batch([260], 2, 1, 64, std=0.3)
        b.q[:, :, 0] = 1.0
        b.k[blocked, 0, 0] = -math.inf
        b.forward()
        n = 260
        for h in range(2):
            z = (b.q[:, h].to(F64) @ b.k[:, 0].to(F64).T) * b.scale
            z = z.masked_fill(~torch.ones(n, n, dtype=torch.bool, device=DEV).tril_(), -math.inf)
            want = torch.softmax(z, 1) @ b.v[:, 0].to(F64)
            none = want.isnan().all(1)                      # queries that see no other key: 0 / 0 by the formula
            got = b.out[:, h].to(F64)
            assert bool(got[none].isnan().all()) and not bool(got[~none].isnan().any())
            assert float((got[~none] - want[~none]).abs().max()) <= 2 * U[BF16] * float(b.v.abs().max())


def test_attention_does_not_see_what_lies_behind_a_key():
    # a NaN or infinity in a later key changes nothing for the queries in front of it
    a, b = Batch([400], 2, 1, 128), Batch([400], 2, 1, 128)
    b.k[300, 0] = float("nan")
    b.k[301, 0] = math.inf
    a.forward()
    b.forward()
    assert same_bits(a.out[:300], b.out[:300]) and torch.equal(a.lse[:, :300], b.lse[:, :300])
    assert bool(b.out[300:].isnan().all())


def test_sequences_do_not_see_each_other():
    a = Batch([130, 70, 200], 4, 2, 64)
    b = Batch([130, 70, 200], 4, 2, 64)
    for t in (b.q, b.k, b.v, b.dout):
        t[130:200] = float("nan")
    for x in (a, b):
        x.forward()
        x.backward()
    for s in (slice(0, 130), slice(200, 400)):
        assert same_bits(a.out[s], b.out[s]) and torch.equal(a.lse[:, s], b.lse[:, s])
        for g, w in zip(b.grads, a.grads):
            assert same_bits(g[s].contiguous(), w[s].contiguous())


def test_attention_gradient_is_the_derivative_of_the_formula():
    b = Batch([90, 140], 4, 2, 64, std=0.7)
    b.forward()
    b.backward()
    x = [t.to(F64) for t in (b.q, b.k, b.v)]
    d = [normal(20 + i, t.shape).to(F64) for i, t in enumerate(x)]

    def value(t):
        q, k, v = (a + t * s for a, s in zip(x, d))
        total = 0.0
        for rows, h, kh in b.pieces():
            n = q[rows].shape[0]
            z = (q[rows, h] @ k[rows, kh].T) * b.scale
            z = z.masked_fill(~torch.ones(n, n, dtype=torch.bool, device=DEV).tril_(), -math.inf)
            total += float(((torch.softmax(z, 1) @ v[rows, kh]) * b.dout[rows, h].to(F64)).sum())
        return total

    t = 1e-4
    want = (value(t) - value(-t)) / (2 * t)
    got = sum(float((g.to(F64) * s).sum()) for g, s in zip(b.grads, d))
    # each element is good to about two bf16 roundings, of either sign
    room = 4 * U[BF16] * math.sqrt(sum(float((g.to(F64) * s).square().sum()) for g, s in zip(b.grads, d))) + 1e-5 * abs(want)
    assert abs(got - want) <= 4 * room


def test_attention_gives_the_same_bits_every_time_and_on_another_stream():
    b = Batch([1000, 300, 17], 8, 2, 128)
    b.forward()
    b.backward()
    first = [t.clone() for t in (b.out, b.lse, *b.grads)]
    side = torch.cuda.Stream()
    for stream in (None, side):
        for t in (b.out, b.lse, *b.grads):
            t.fill_(0)
        torch.cuda.synchronize()
        b.forward(stream)
        ws = workspace(dte.dte_attention_backward_workspace_bytes(b.tokens, b.hq))
        torch.cuda.synchronize()
        b.backward(stream, ws)
        torch.cuda.synchronize()
        for t, w in zip((b.out, b.lse, *b.grads), first):
            assert same_bits(t, w)


def test_attention_captured_and_replayed_on_other_lengths():
    b = Batch([200, 312], 4, 2, 128)
    other = Batch([1, 400, 111], 4, 2, 128, seed=30)
    starts = torch.empty(4, dtype=torch.int32, device=DEV)
    plan = workspace(dte.dte_attention_plan_bytes(512, 3))
    ws = workspace(dte.dte_attention_backward_workspace_bytes(512, 4))

    def step():
        dte.dte_attention_plan(starts, 512, plan)
        dte.dte_attention_forward(b.q, b.k, b.v, plan, b.out, b.lse)
        dte.dte_attention_backward(b.q, b.k, b.v, b.out, b.lse, b.dout, plan, *b.grads, ws)

    starts.copy_(torch.tensor([0, 200, 512, 512]))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    b.check_forward()
    b.check_backward()
    starts.copy_(other.starts)
    for name in ("q", "k", "v", "dout"):
        getattr(b, name).copy_(getattr(other, name))
    b.lengths = other.lengths
    graph.replay()
    b.check_forward()
    b.check_backward()


def test_attention_of_nothing_and_without_lse():
    b = Batch([], 2, 1, 64, front=0, behind=9)
    b.forward()
    b.backward()
    b.check_forward()
    b.check_backward()
    e = Batch([], 2, 1, 64)
    e.forward()
    e.backward()
    a = Batch([40, 9], 2, 1, 64)
    a.forward()
    out = a.out.clone()
    a.out.zero_()
    dte.dte_attention_forward(a.q, a.k, a.v, a.plan, a.out, None)
    assert same_bits(a.out, out)


@pytest.mark.parametrize("starts", [[0, 50, 40, 100], [0, 101], [-1, 100], [5, 2], [0, 2 ** 40]])
def test_bad_starts_set_the_flag_and_leave_the_outputs(starts):
    b = Batch([100], 2, 1, 64)
    b.out.fill_(3.0)
    flags = torch.zeros(1, dtype=torch.int64, device=DEV)
    b.plan = plan_of(torch.tensor(starts, dtype=torch.int64, device=DEV), 100, flags)
    assert int(flags) == dte.DTE_DEV_BOUNDS
    b.forward()
    b.backward()
    for t in (b.out, b.lse, *b.grads):
        assert bool((t == 3.0).all())


def test_a_plan_of_another_batch_sets_the_flag_and_leaves_the_outputs():
    b, c = Batch([100], 2, 1, 64), Batch([100], 2, 1, 64, behind=1)
    for plan in (c.plan, torch.zeros(4096, dtype=torch.uint8, device=DEV), b.plan[:256]):
        flags = torch.zeros(1, dtype=torch.int64, device=DEV)
        dte.dte_attention_forward(b.q, b.k, b.v, plan, b.out, b.lse, flags=flags)
        dte.dte_attention_backward(b.q, b.k, b.v, b.out, b.lse, b.dout, plan, *b.grads,
                                   workspace(dte.dte_attention_backward_workspace_bytes(100, 2)), flags=flags)
        assert int(flags) == dte.DTE_DEV_BOUNDS
        for t in (b.out, b.lse, *b.grads):
            assert bool((t == 3.0).all())


def test_attention_beyond_32_bit_offsets():
    rows, ld = 40000, 2 ** 17                              # 5.2 G elements between the first row and the last
    buf = torch.empty(rows, ld, dtype=BF16, device=DEV)
    x = buf[:, :6 * 64].unflatten(1, (6, 64))
    small = Batch([39000, 1000], 1, 1, 64, seed=9)
    x[:, 0], x[:, 1], x[:, 2] = small.q[:, 0], small.k[:, 0], small.v[:, 0]
    x[:, 3], x[:, 4] = small.dout[:, 0], 3.0
    small.forward()
    small.backward()
    lse = torch.empty_like(small.lse)
    dte.dte_attention_forward(x[:, 0:1], x[:, 1:2], x[:, 2:3], small.plan, x[:, 4:5], lse)
    assert same_bits(x[:, 4:5].contiguous(), small.out) and torch.equal(lse, small.lse)
    grads = [torch.empty_like(g) for g in small.grads]
    dte.dte_attention_backward(x[:, 0:1], x[:, 1:2], x[:, 2:3], x[:, 4:5], lse, x[:, 3:4], small.plan, grads[0], x[:, 5:6], grads[2],
                               workspace(dte.dte_attention_backward_workspace_bytes(rows, 1)))
    assert same_bits(x[:, 5:6].contiguous(), small.grads[1]) and same_bits(grads[0], small.grads[0]) and same_bits(grads[2], small.grads[2])


# ---- gradient norm and clipping ---------------------------------------------------------------------------------

def views(seed, sizes, dtype, std=1.0):
    """Tensors of the given sizes; every third starts at an odd element."""
    out = []
    for i, n in enumerate(sizes):
        t = normal(seed + i, (n + 1,), std, dtype)
        out.append(t[1:] if i % 3 == 1 else t[:n])
    return out


def squares(tensors):
    return sum((float(t.to(F64).square().sum()) for t in tensors), 0.0)


def norm_of(tensors, max_norm, outs=None, accumulate=None):
    total = torch.full((), float("nan") if accumulate is None else accumulate, dtype=F64, device=DEV)
    norm = torch.empty((), device=DEV)
    dte.dte_grad_sum_squares(tensors, total, workspace(dte.dte_grad_sum_squares_workspace_bytes(len(tensors))), accumulate=accumulate is not None)
    dte.dte_grad_clip(tensors, total, max_norm, norm, outs)
    return float(total), float(norm)


SUM_REL = 14 * E        # 8 squares in a row, two joins, a square's own rounding; everything else in 64 bits
SIZES = [[1], [0, 3], [7, 8, 9], [16383, 16384, 16385, 5], [100000, 1, 0, 8191, 4096], [1 << 20, 12345]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda v: "-".join(map(str, v)))
@pytest.mark.parametrize("src", [F32, BF16])
@pytest.mark.parametrize("dst", [F32, BF16, None])
def test_clip(sizes, src, dst):
    for max_norm in (0.37, 1e9):
        g = views(1, sizes, src)
        before = [t.clone() for t in g]
        outs = None if dst is None else [t[:n] for t, n in zip(views(50, sizes, dst), sizes)]
        total, norm = norm_of(g, max_norm, outs)
        want = squares(before)
        assert abs(total - want) <= SUM_REL * want
        assert abs(norm - math.sqrt(total)) <= E * norm
        f = min(1.0, max_norm / math.sqrt(total)) if total else 1.0
        for t, o, b in zip(g, g if outs is None else outs, before):
            if f == 1.0 and o.dtype == b.dtype:
                assert same_bits(o, b)
            w = b.to(F64) * f
            assert_within(o, w, (U[o.dtype] * 1.01 + 3 * E) * w.abs() + 1e-38, "clipped")
            if outs is not None:
                assert same_bits(t, b)


def test_norm_of_many_tensors_adds_to_what_is_there_and_gives_the_same_bits():
    g = views(3, [(i * 37) % 900 for i in range(2500)], BF16, 1e-3)
    want = squares(g)
    a, _ = norm_of(g, 1e9)
    b, _ = norm_of(g, 1e9)
    c, norm = norm_of(g, 1e9, accumulate=2.5)
    assert a == b and abs(a - want) <= SUM_REL * want
    assert abs(c - (2.5 + want)) <= SUM_REL * want + 1e-15
    before = [t.clone() for t in g]
    norm_of(g, 0.5 * math.sqrt(want))
    for t, w in zip(g, before):
        assert_within(t, w.to(F64) * 0.5, (U[BF16] * 1.01 + 14 * E) * w.to(F64).abs() + 1e-38, "half")


@pytest.mark.parametrize("size", [1e-30, 1e-25, 1e25, 1e30, 3e38])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_squares_beyond_fp32(size, dtype):
    g = [torch.full((n,), size, dtype=dtype, device=DEV) for n in (40000, 3, 8)]
    want = squares(g)
    total, norm = norm_of(g, 1e300)
    assert abs(total - want) <= SUM_REL * want
    if math.sqrt(want) < 3e38:
        assert abs(norm - math.sqrt(want)) <= 8 * E * norm
        norm_of(g, math.sqrt(want) / 4)
        w = torch.full((3,), size, dtype=dtype).to(F64).to(DEV) / 4
        assert_within(g[1], w, (U[dtype] * 1.01 + 16 * E) * w, "a quarter")


def test_large_and_small_gradients_together():
    g = [torch.full((5000,), 1e-30, device=DEV), torch.full((100,), 2.0, device=DEV), torch.zeros(70000, device=DEV)]
    total, norm = norm_of(g, 100.0)
    assert total == 400.0 and norm == 20.0


@pytest.mark.parametrize("bad", [float("nan"), math.inf, -math.inf])
def test_a_norm_that_is_not_finite_leaves_the_gradients(bad):
    g = views(5, [5000, 33, 9], F32)
    g[1][7] = bad
    before = [t.clone() for t in g]
    _, norm = norm_of(g, 1e-3)
    assert not math.isfinite(norm)
    for t, b in zip(g, before):
        assert same_bits(t, b)


def test_no_tensors_and_no_elements():
    assert norm_of([], 1.0) == (0.0, 0.0)
    assert norm_of([torch.empty(0, device=DEV)], 1.0) == (0.0, 0.0)
    assert norm_of([], 1.0, accumulate=9.0) == (9.0, 3.0)


def test_clip_beyond_32_bit_offsets():
    n = 2 ** 32 + 12345
    g = torch.zeros(n, dtype=BF16, device=DEV)
    for at in (0, 2 ** 32 - 1, 2 ** 32 + 7, n - 1):
        g[at] = 2.0
    total, norm = norm_of([g], 1.0)
    assert total == 16.0 and norm == 4.0
    for at in (0, 2 ** 32 - 1, 2 ** 32 + 7, n - 1):
        assert float(g[at]) == 0.5


def test_clip_captured_and_replayed():
    g = views(7, [5000, 33, 9], F32)
    outs = [torch.empty_like(t) for t in g]
    total, norm = torch.empty((), dtype=F64, device=DEV), torch.empty((), device=DEV)
    ws = workspace(dte.dte_grad_sum_squares_workspace_bytes(3))

    def step():
        dte.dte_grad_sum_squares(g, total, ws)
        dte.dte_grad_clip(g, total, 1.0, norm, outs)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for scale in (1.0, 3.0):
        for t in g:
            t.mul_(scale)
        graph.replay()
        want = math.sqrt(squares(g))
        assert abs(float(norm) - want) <= 8 * E * want
        for t, o in zip(g, outs):
            assert_within(o, t.to(F64) / want, 16 * E * t.to(F64).abs() + 1e-38, "replayed")


# ---- waits that run out -------------------------------------------------------------------------------------------

def test_a_wait_that_runs_out_sets_the_flag_and_leaves_the_device_usable():
    for hq, hk, dim, lengths in ((4, 2, 128, [700, 90]), (3, 3, 64, [400])):
        b = Batch(lengths, hq, hk, dim)
        ws = workspace(dte.dte_attention_backward_workspace_bytes(b.tokens, hq))
        b.forward()
        dte.lib().dte_attention_set_wait_limit(1)             # every wait that is not over at once gives up
        try:
            flags = torch.zeros(2, dtype=torch.int64, device=DEV)
            dte.dte_attention_forward(b.q, b.k, b.v, b.plan, torch.empty_like(b.out), None, flags=flags[:1])
            dte.dte_attention_backward(b.q, b.k, b.v, b.out, b.lse, b.dout, b.plan, *(torch.empty_like(g) for g in b.grads), ws, flags=flags[1:])
            torch.cuda.synchronize()
        finally:
            dte.lib().dte_attention_set_wait_limit(0)
        assert flags.tolist() == [dte.DTE_DEV_TIMEOUT] * 2
        b.forward()
        b.check_forward()
        b.backward()
        b.check_backward()


def test_a_gradient_of_cut_heads_that_gave_up_leaves_nothing_for_the_next_one():
    b = Batch([640], 16, 1, 64)
    ws = workspace(dte.dte_attention_backward_workspace_bytes(b.tokens, 16))
    b.forward()
    b.backward(None, ws)
    want = [g.clone() for g in b.grads]
    dte.lib().dte_attention_set_wait_limit(1)
    try:
        flags = torch.zeros(1, dtype=torch.int64, device=DEV)
        dte.dte_attention_backward(b.q, b.k, b.v, b.out, b.lse, b.dout, b.plan, *(torch.empty_like(g) for g in b.grads), ws, flags=flags)
        torch.cuda.synchronize()
    finally:
        dte.lib().dte_attention_set_wait_limit(0)
    assert flags.tolist() == [dte.DTE_DEV_TIMEOUT]
    b.backward(None, ws)
    for g, w in zip(b.grads, want):
        assert same_bits(g, w)


def test_gradients_of_cut_heads_on_two_streams():
    batches = [Batch([900, 30], 32, 1, 128, seed=s) for s in (1, 60)]
    spaces = [workspace(dte.dte_attention_backward_workspace_bytes(930, 32)) for _ in batches]
    want = []
    for b, ws in zip(batches, spaces):
        b.forward()
        b.backward(None, ws)
        want.append([g.clone() for g in b.grads])
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for _ in range(10):
        for b, s, ws in zip(batches, streams, spaces):
            b.backward(s, ws)
    torch.cuda.synchronize()
    for b, w in zip(batches, want):
        for g, x in zip(b.grads, w):
            assert same_bits(g, x)


def test_attention_on_two_streams_with_one_plan():
    a, b = Batch([500, 300], 4, 2, 128), Batch([500, 300], 4, 2, 128, seed=40)
    b.plan = a.plan
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [workspace(dte.dte_attention_backward_workspace_bytes(800, 4)) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s, ws in zip((a, b), streams, spaces):
            x.forward(s)
            x.backward(s, ws)
    torch.cuda.synchronize()
    for x in (a, b):
        x.check_forward()
        x.check_backward()


def test_work_behind_the_gradient_in_the_stream_sees_all_of_it():
    # the passes overlap inside the call; what follows in the stream must find both finished
    b = Batch([1500, 700, 40], 8, 2, 64)
    b.forward()
    b.backward()
    want = [g.clone() for g in b.grads]
    for _ in range(20):
        for g in b.grads:
            g.zero_()
        b.backward()
        got = [g + 0 for g in b.grads]
        for g, w in zip(got, want):
            assert same_bits(g, w)
