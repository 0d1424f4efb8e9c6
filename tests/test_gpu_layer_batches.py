"""The operators inside and behind the layers at the sizes of batches: launches that small tests do not reach, calls one behind
the other on one workspace, values at the ends of the types' ranges.  Tolerances as in test_gpu_layer_operators."""
import math

import pytest
import torch

import paper_2608_00455_b200 as dte
from test_gpu_layer_operators import BF16, DEV, E, F32, F64, U, Batch, assert_within, norm_of, normal, same_bits, squares, workspace

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
