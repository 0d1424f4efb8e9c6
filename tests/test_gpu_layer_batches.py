"""The operators inside and behind the layers at the sizes of batches: launches that small tests do not reach, calls one behind
the other on one workspace, values at the ends of the types' ranges.  Tolerances as in test_gpu_layer_operators."""
import math

import pytest
import torch

import paper_2608_00455_b200 as dte
from test_gpu_layer_operators import (BF16, DEV, E, F32, F64, U, Batch, assert_within, gen, heads_of, norm_of, normal, rope_want, same_bits,
                                      squares, workspace)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,hq,hk,dim", [([1500, 700, 40], 8, 2, 64), ([900, 30], 32, 1, 128), ([130] * 40, 4, 4, 64)])
def test_gradients_one_behind_the_other_on_one_workspace(lengths, hq, hk, dim):
    # delta and the counters of the call in front are still in the workspace: with other inputs they would show
    b = Batch(lengths, hq, hk, dim)
    b.forward()
    douts = [b.dout, normal(90, b.dout.shape, 3.0, b.dout.dtype)]
    want = []
    for d in douts:
        b.dout = d
        b.backward()
        b.check_backward()
        want.append([g.clone() for g in b.grads])
    ws = workspace(dte.dte_attention_backward_workspace_bytes(b.tokens, hq))
    got = [[torch.empty_like(g) for g in b.grads] for _ in range(20)]
    for i, g in enumerate(got):
        b.dout, b.grads = douts[i % 2], g
        b.backward(None, ws)
    for i, g in enumerate(got):
        for t, w in zip(g, want[i % 2]):
            assert same_bits(t, w)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("into", [None, F32, BF16])
def test_a_norm_beyond_fp32_is_shown_as_infinite_and_leaves_the_gradients(dtype, into):
    g = [torch.full((n,), 3e38, dtype=dtype, device=DEV) for n in (40000, 3, 8)]
    before = [t.clone() for t in g]
    outs = None if into is None else [torch.empty(t.shape, dtype=into, device=DEV) for t in g]
    total, norm = norm_of(g, 1.0, outs)
    assert math.isfinite(total) and norm == math.inf
    for t, o, b in zip(g, g if outs is None else outs, before):
        assert same_bits(t, b) and same_bits(o, b.to(o.dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("into", [None, F32, BF16])
@pytest.mark.parametrize("ratio", [0.7, 2.0 ** -125, 1e-38, 2.0 ** -126, 1e-40, 1e-44, 1e-50, 1e-70])
def test_clipping_by_any_factor(dtype, into, ratio):
    # gradients of all sizes beside some that are as large as the norm
    g = [normal(5, (40001,), 1e35, dtype), normal(6, (3,), 1e36, dtype), normal(7, (9000,), 1.0, dtype)]
    before = [t.clone() for t in g]
    outs = None if into is None else [torch.empty(t.shape, dtype=into, device=DEV) for t in g]
    max_norm = math.sqrt(squares(g)) * ratio
    total, norm = norm_of(g, max_norm, outs)
    assert math.isfinite(norm)
    for t, o, b in zip(g, g if outs is None else outs, before):
        w = b.to(F64) * (max_norm / math.sqrt(total))
        # the quotient and the product in fp32, the output's rounding; below 2^-126 in steps of 2^-149 (fp32) or 2^-133 (bf16)
        step = 2.0 ** -149 if o.dtype == F32 else 2.0 ** -133
        assert_within(o, w, (U[o.dtype] + 3 * E) * w.abs() + 0.51 * step + 2.0 ** -149, f"{ratio}")


# ---- rotary positions: from 1184 tokens on (eight for each of 148 multiprocessors) a CTA holds two of them ------------

@pytest.mark.parametrize("tokens", [1183, 1184, 1185, 2501])
@pytest.mark.parametrize("dim,rot,extra,offset", [(128, 128, 0, 0), (64, 32, 8, 8), (66, 34, 2, 2), (9, 6, 3, 1), (6, 6, 0, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rope_of_a_batch(tokens, dim, rot, extra, offset, interleaved, dtype):
    freq = (10000.0 ** (-torch.arange(rot // 2, dtype=F64) * 2 / rot)).to(DEV)
    q, k = heads_of(1, tokens, 5, dim, dtype, extra, offset), heads_of(2, tokens, 2, dim, dtype, extra, offset)
    pos = torch.randint(0, 200000, (tokens,), generator=gen(3), device=DEV)
    pos[0], pos[3], pos[6:8], pos[-1] = -1, -1, -1, 0                # padding at either place of a CTA, and at both
    outs = [heads_of(4, tokens, t.shape[1], dim, dtype, extra, offset) for t in (q, k)]
    for inverse in (False, True):
        dte.dte_rope(q, k, pos, freq, *outs, interleaved=interleaved, amplitude=1.25, inverse=inverse)
        for t, o in zip((q, k), outs):
            want, bound = rope_want(t, pos, freq, interleaved, 1.25, inverse)
            assert_within(o[..., :rot], want[..., :rot], bound[..., :rot] + U[dtype] * 1.01 * want[..., :rot].abs() + 1e-38, f"{tokens}")
            assert same_bits(o[..., rot:].contiguous(), t[..., rot:].contiguous())
            for i in (0, 3, 6, 7):
                assert same_bits(o[i].contiguous(), t[i].contiguous())
    dte.dte_rope(q, k, pos, freq, interleaved=interleaved, amplitude=1.25, inverse=True)
    for t, o in zip((q, k), outs):
        assert same_bits(t.contiguous(), o.contiguous())


@pytest.mark.parametrize("dim", [256, 260])
def test_rope_of_as_many_heads_as_a_call_takes(dim):
    # odd rows and 4095 heads: at 256 columns the numbers of a CTA's pieces are just small enough for two tokens, at 260 for one
    tokens, heads = 1185, 4095
    freq = (10000.0 ** (-torch.arange(128, dtype=F64) / 128)).to(DEV)
    q = heads_of(1, tokens, heads, dim, BF16, 1, 1)
    pos = torch.randint(0, 200000, (tokens,), generator=gen(3), device=DEV)
    pos[5] = -1
    out = torch.zeros(tokens, heads * dim + 1, dtype=BF16, device=DEV)[:, :heads * dim].unflatten(1, (heads, dim))
    dte.dte_rope(q, None, pos, freq, out)
    for a in range(0, tokens, 100):                   # few tokens at a time: the other launch
        b = min(a + 100, tokens)
        part = torch.zeros(b - a, heads, dim, dtype=BF16, device=DEV)
        dte.dte_rope(q[a:b], None, pos[a:b], freq, part)
        assert same_bits(out[a:b].contiguous(), part)


def test_rope_beyond_32_bit_offsets():
    rows, ld = 40000, 2 ** 17                         # 5.2 G elements between the first row and the last
    buf = torch.empty(rows, ld, dtype=BF16, device=DEV)
    x = buf[:, ld - 5 * 64:].unflatten(1, (5, 64))
    x.copy_(normal(1, (rows, 5, 64), 1.0, BF16))
    want = x.contiguous()
    freq = (10000.0 ** (-torch.arange(32, dtype=F64) / 32)).to(DEV)
    pos = torch.arange(rows, device=DEV)
    dte.dte_rope(x[:, :4], x[:, 4:], pos, freq)
    dte.dte_rope(want[:, :4], want[:, 4:], pos, freq)
    assert same_bits(x.contiguous(), want)
    x.zero_()
    dte.dte_rope(want, None, pos, freq, x, inverse=True)
    back = torch.empty_like(want)
    dte.dte_rope(want, None, pos, freq, back, inverse=True)
    assert same_bits(x.contiguous(), back)


# ---- attention: several pieces of work for every CTA --------------------------------------------------------------

@pytest.mark.parametrize("lengths,hq,hk,dim", [([700, 129, 1, 256, 0, 300, 640, 128, 1025, 77, 383], 32, 8, 128),        # 560 pieces of two heads
                                               ([1300, 5, 900, 257, 640], 32, 4, 128),
                                               ([200] * 12 + [1, 2, 385], 16, 16, 64), ([900, 1000, 31], 9, 3, 40),      # pairs of tiles of a head
                                               ([450, 700, 129], 48, 6, 96)])
def test_attention_of_a_batch(lengths, hq, hk, dim):
    b = Batch(lengths, hq, hk, dim, front=2, behind=70, fused=True)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()
    first = [t.clone() for t in (b.out, b.lse)]
    b.out.fill_(3.0)
    b.lse.fill_(3.0)
    b.forward()
    for t, w in zip((b.out, b.lse), first):
        assert same_bits(t, w)


def test_attention_of_thousands_of_short_sequences():
    lengths = torch.randint(0, 12, (3000,), generator=torch.Generator().manual_seed(5)).tolist() + [400]
    b = Batch(lengths, 2, 1, 64, behind=3)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


def test_scores_that_differ_from_piece_to_piece_of_a_cta():
    # maxima of very different size in heads and sequences that one CTA works on in turn: nothing of a piece may stay for the next
    b = Batch([300] * 10 + [140] * 10, 32, 8, 64)
    b.q.mul_(torch.logspace(-2, 2, 32, device=DEV).to(BF16)[None, :, None])
    b.v.mul_(torch.logspace(-3, 3, b.tokens, device=DEV).to(BF16)[:, None, None])
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()
