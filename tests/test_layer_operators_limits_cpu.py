"""Arguments of rotary positions, attention and clipping at the ends of what their types hold: refused, or answered right, without a GPU."""
import math

import pytest
import torch

import paper_2608_00455_b200 as dte
from paper_2608_00455_b200 import operators as ops
from test_layer_operators_cpu import forward, refused

SMALLEST = 2.0 ** -126          # of fp32's normal numbers; half a step below it, 2^-126 - 2^-150, is a tie that rounds up to it


@pytest.mark.parametrize("scale", [1e-300, 1e-46, 1e-39, SMALLEST * (1 - 2.0 ** -23)])
def test_attention_refuses_a_scale_that_fp32_cannot_hold(scale):
    refused(forward(scale=scale), "scale")


@pytest.mark.parametrize("scale", [SMALLEST, SMALLEST * (1 - 2.0 ** -24), 1e-3, 2e38])
def test_attention_takes_every_scale_that_fp32_holds(scale):
    refused(forward(scale=scale), "device")          # everything else is in order


@pytest.fixture
def on_the_host(monkeypatch):
    """Tensors on the CPU pass for a device's (ordinal -1, which the library refuses last of all): the binding's own checks alone."""
    monkeypatch.setattr(ops, "_device", lambda t, name: -1)
    monkeypatch.setattr(ops, "_stream", lambda stream, device: None)


def test_heads_without_columns_are_refused(on_the_host):
    x, t, f, b = torch.zeros(4, 1, 0), torch.zeros(4, dtype=torch.int64), torch.ones(4, dtype=torch.float64), torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda: dte.dte_rope(x, None, t, f), lambda: dte.dte_attention_forward(x, x, x, b, x, None),
                 lambda: dte.dte_attention_backward(x, x, x, x, torch.zeros(1, 4), x, b, x, x, x, b)):
        with pytest.raises(dte.DteError, match="head_dim") as e:
            call()
        assert e.value.status == 1


def test_outputs_of_rotary_positions_have_their_inputs_shapes(on_the_host):
    # two heads of 8 columns have the columns of one head of 16, and are something else
    q, k, t, f = torch.zeros(4, 2, 8), torch.zeros(4, 4, 8), torch.zeros(4, dtype=torch.int64), torch.ones(4, dtype=torch.float64)
    for outs, word in (((torch.zeros(4, 1, 16), None), "q_out"), ((torch.zeros(4, 4, 4), None), "q_out"), ((None, torch.zeros(4, 2, 16)), "k_out"),
                       ((torch.zeros(2, 4, 8), None), "q_out")):
        with pytest.raises(dte.DteError, match=f"{word} must have") as e:
            dte.dte_rope(q, k, t, f, *outs)
        assert e.value.status == 1
    with pytest.raises(dte.DteError, match="device"):          # everything else is in order
        dte.dte_rope(q, k, t, f, torch.zeros(4, 2, 8), torch.zeros(4, 4, 8))


@pytest.mark.parametrize("rot,base,positions", [(128, 1e6, 6.0), (128, 1e6, 2.0), (2, 1e4, 1.0), (64, 1e4, 6.28)])
def test_a_ramp_where_no_pair_turns_once(rot, base, positions):
    # the fastest pair turns positions / (2 pi) times, fewer than slow_turns = 1: every pair is squeezed, the fastest too
    plain, _ = dte.dte_rope_frequencies(rot, base)
    f, _ = dte.dte_rope_frequencies(rot, base, dte.DTE_ROPE_RAMP, 4.0, positions)
    assert positions / (2 * math.pi) < 1
    assert torch.equal(f, plain / 4)


def test_a_ramp_where_every_pair_turns_often():
    plain, _ = dte.dte_rope_frequencies(8, 10.0)
    f, _ = dte.dte_rope_frequencies(8, 10.0, dte.DTE_ROPE_RAMP, 4.0, 1e9)
    assert torch.equal(f, plain)


@pytest.mark.parametrize("args", [(4, 1e200, dte.DTE_ROPE_BASE, 1e60), (128, 1e308, dte.DTE_ROPE_BASE, 4.0)])
def test_a_changed_base_beyond_fp64_is_refused(args):
    with pytest.raises(dte.DteError, match="base") as e:
        dte.dte_rope_frequencies(*args)
    assert e.value.status == 1
