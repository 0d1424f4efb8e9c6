"""The operators inside and behind the layers at the sizes of batches: launches that small tests do not reach, calls one behind
the other on one workspace, values at the ends of the types' ranges.  Tolerances as in test_gpu_layer_operators."""
import math

import pytest
import torch

import paper_2608_00455_b200 as dte
from test_gpu_layer_operators import BF16, DEV, F32, Batch, norm_of, normal, same_bits, squares, workspace

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
