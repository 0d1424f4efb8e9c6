"""Arguments of rotary positions, attention and clipping at the ends of what their types hold: refused, or answered right, without a GPU."""
import pytest

import paper_2608_00455_b200 as dte
from test_layer_operators_cpu import forward, refused

SMALLEST = 2.0 ** -126          # of fp32's normal numbers; half a step below it, 2^-126 - 2^-150, is a tie that rounds up to it


@pytest.mark.parametrize("scale", [1e-300, 1e-46, 1e-39, SMALLEST * (1 - 2.0 ** -23)])
def test_attention_refuses_a_scale_that_fp32_cannot_hold(scale):
    refused(forward(scale=scale), "scale")


@pytest.mark.parametrize("scale", [SMALLEST, SMALLEST * (1 - 2.0 ** -24), 1e-3, 2e38])
def test_attention_takes_every_scale_that_fp32_holds(scale):
    refused(forward(scale=scale), "device")          # everything else is in order
