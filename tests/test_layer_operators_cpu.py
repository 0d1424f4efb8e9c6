"""Host side of rotary positions, attention and gradient clipping, without a GPU: frequencies, sizes of plans and workspaces, and
arguments that are refused before any CUDA call."""
import math
import struct

import pytest
import torch

import paper_2608_00455_b200 as dte
from paper_2608_00455_b200 import operators as ops

UNFIT = 2 ** 64 - 1


def matrix(rows, cols, ld=None, dtype=ops.DTE_BF16, data=4096):
    return ops._pack_matrix(data, rows, cols, cols if ld is None else ld, dtype, 0)


def ids(count, dtype=ops.DTE_I64, data=8192):
    return ops._pack_ids(data, count, dtype, 0)


def tensor(numel, dtype=ops.DTE_F32, data=4096):
    return ops._pack_ids(data, numel, dtype, 0)        # the same fields


def refused(status, word):
    assert status == 1
    assert word in dte.lib().dte_last_error().decode()


# ---- frequencies ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 1e6), (128, 1e6), (1024, 500000.0)])
def test_frequencies(rot, base):
    plain = [base ** (-2 * i / rot) for i in range(rot // 2)]

    def close(got, want):
        assert len(got) == len(want) and all(abs(g - w) <= 8 * 2.0 ** -53 * rot * abs(w) for g, w in zip(got.tolist(), want))

    f, a = dte.dte_rope_frequencies(rot, base)
    assert a == 1.0 and f.dtype == torch.float64 and float(f[0]) == 1.0
    close(f, plain)
    f, a = dte.dte_rope_frequencies(rot, base, dte.DTE_ROPE_LINEAR, 4.0)
    assert a == 1.0
    close(f, [x / 4 for x in plain])
    if rot > 2:
        f, a = dte.dte_rope_frequencies(rot, base, dte.DTE_ROPE_BASE, 4.0)
        assert a == 1.0 and float(f[0]) == 1.0
        assert abs(float(f[-1]) * 4.0 / plain[-1] - 1) < 1e-12          # the slowest pair is stretched by the whole factor
    f, a = dte.dte_rope_frequencies(rot, base, dte.DTE_ROPE_RAMP, 4.0, 32768.0)
    assert abs(a - (0.1 * math.log(4.0) + 1)) < 1e-15
    for x, p in zip(f.tolist(), plain):
        turns = 32768 * p / (2 * math.pi)
        assert p / 4 * (1 - 1e-12) <= x <= p * (1 + 1e-12)
        step = base ** (2 / rot)                                        # one index of the ramp's rounding outwards
        if turns > 32.0 * step:
            assert abs(x / p - 1) < 1e-12
        if turns < 1.0 / step:
            assert abs(x * 4 / p - 1) < 1e-12


def test_a_factor_of_one_changes_nothing():
    plain, _ = dte.dte_rope_frequencies(128, 1e6)
    for kind in (dte.DTE_ROPE_LINEAR, dte.DTE_ROPE_BASE, dte.DTE_ROPE_RAMP):
        f, a = dte.dte_rope_frequencies(128, 1e6, kind, 1.0, 4096.0)
        assert a == 1.0 and float((f / plain - 1).abs().max()) < 1e-15


@pytest.mark.parametrize("args,word", [((0, 1e4), "rot"), ((7, 1e4), "rot"), ((1026, 1e4), "rot"), ((8, 1.0), "base"),
                                       ((8, float("nan")), "base"), ((8, math.inf), "base"), ((8, 1e4, 4), "scaling"),
                                       ((8, 1e4, 1, 0.5), "factor"), ((8, 1e4, 2, math.inf), "factor"), ((2, 1e4, 2, 2.0), "pair"),
                                       ((8, 1e4, 3, 2.0, 0.0), "ramp"), ((8, 1e4, 3, 2.0, 4096.0, 1.0, 2.0), "ramp"),
                                       ((8, 1e4, 3, 2.0, 4096.0, 32.0, 0.0), "ramp"), ((-2, 1e4), "negative")])
def test_frequencies_refuse(args, word):
    with pytest.raises(dte.DteError, match=word):
        dte.dte_rope_frequencies(*args)


# ---- refusals ---------------------------------------------------------------------------------------------------

def rope(q=matrix(4, 64), k=None, dim=16, pos=ids(4), freq=4096, rot=16, layout=0, amplitude=1.0, qo=matrix(4, 64, data=1 << 20), ko=None,
         device=-1):
    return dte.lib().dte_rope(q, k, dim, pos, freq, rot, layout, amplitude, 0, qo, ko, device, None)


def test_rope_refuses():
    refused(rope(), "device")                       # everything else is in order
    refused(rope(q=None), "q is null")
    refused(rope(qo=None), "q_out is null")
    refused(rope(k=matrix(4, 64)), "k_out is null")
    refused(rope(ko=matrix(4, 64)), "k is null")
    refused(rope(pos=None), "ids are null")
    refused(rope(pos=ids(4, dtype=ops.DTE_F32)), "DTE_I32 or DTE_I64")
    for rot, dim in ((0, 16), (3, 16), (18, 16), (2, 0), (2, 1026)):
        refused(rope(rot=rot, dim=dim), "rot")
    refused(rope(dim=24, rot=8), "multiple of head_dim")
    refused(rope(layout=2), "layout")
    refused(rope(amplitude=1e39), "amplitude")
    refused(rope(amplitude=float("nan")), "amplitude")
    refused(rope(freq=None), "frequencies")
    refused(rope(freq=4100), "frequencies")
    refused(rope(pos=ids(5)), "one row per position")
    refused(rope(qo=matrix(4, 32)), "same columns")
    refused(rope(qo=matrix(4, 64, dtype=ops.DTE_F32, data=1 << 20)), "one type")
    refused(rope(k=matrix(4, 16, dtype=ops.DTE_F32), ko=matrix(4, 16, dtype=ops.DTE_F32)), "one type")
    refused(rope(qo=matrix(4, 64, ld=63)), "overlap")
    refused(rope(qo=matrix(4, 64, ld=72)), "in place")
    refused(rope(q=matrix(4, 16 * 4096), qo=matrix(4, 16 * 4096, data=1 << 20)), "4095 heads")


def forward(q=matrix(300, 512), k=matrix(300, 128), v=matrix(300, 128), dim=64, plan=4096, size=1 << 20, scale=0.125, out=matrix(300, 512),
            lse=4096, flags=None, device=-1):
    return dte.lib().dte_attention_forward(q, k, v, dim, plan, size, scale, out, lse, flags, device, None)


def backward(out=matrix(300, 512), lse=4096, dout=matrix(300, 512), dq=matrix(300, 512), dk=matrix(300, 128), dv=matrix(300, 128), ws=4096,
             size=1 << 27, device=-1):
    return dte.lib().dte_attention_backward(matrix(300, 512), matrix(300, 128), matrix(300, 128), 64, out, lse, dout, 4096, 1 << 20, 0.125,
                                            dq, dk, dv, ws, size, None, device, None)


def test_attention_refuses():
    refused(forward(), "device")
    refused(backward(), "device")
    for name, word in (("q", "q is null"), ("k", "k is null"), ("v", "v is null"), ("out", "out is null"), ("plan", "plan")):
        refused(forward(**{name: None}), word)
    for dim in (0, 4, 12, 136):
        refused(forward(dim=dim), "head_dim")
    refused(forward(dim=96), "multiple of head_dim")
    refused(forward(q=matrix(300, 512, dtype=ops.DTE_F32)), "BF16")
    refused(forward(k=matrix(299, 128)), "one row per token")
    refused(forward(v=matrix(300, 64)), "v must have k's")
    refused(forward(k=matrix(300, 192), v=matrix(300, 192)), "multiple of k's heads")
    refused(forward(out=matrix(300, 256)), "q's columns")
    for bad in (matrix(300, 128, data=4104), matrix(300, 128, ld=132), matrix(300, 128, ld=120), matrix(300, 128, ld=0)):
        refused(forward(k=bad), "16-byte aligned")
    refused(forward(out=matrix(300, 512, ld=516)), "16-byte aligned")
    for scale in (0.0, -1.0, float("nan"), math.inf, 3e38):
        refused(forward(scale=scale), "scale")
    refused(forward(plan=4100), "plan")
    refused(forward(size=255), "plan")
    refused(forward(lse=4098), "lse")
    refused(forward(flags=4100), "flags")
    big = 2 ** 24 + 1
    refused(forward(q=matrix(big, 512), k=matrix(big, 128), v=matrix(big, 128)), "2^24 tokens")
    refused(forward(q=matrix(300, 8 * 65536), k=matrix(300, 8), v=matrix(300, 8), dim=8), "heads")
    for name in ("out", "dout", "dq", "dk", "dv"):
        refused(backward(**{name: None}), f"{name} is null")
        refused(backward(**{name: matrix(300, 64)}), "columns")
    refused(backward(lse=None), "lse")
    refused(backward(ws=4097), "256-byte aligned")
    refused(backward(ws=None), "workspace is null")
    assert backward(size=300 * 8 * 4 - 1) == 3


def test_attention_plan_refuses_and_its_size():
    L = dte.lib()
    plan = lambda starts=ids(5), tokens=1000, buf=4096, size=1 << 20, flags=None: L.dte_attention_plan(starts, tokens, buf, size, flags, -1, None)   # noqa: E731
    refused(plan(), "device")
    refused(plan(starts=None), "ids are null")
    refused(plan(starts=ids(0)), "one entry more")
    refused(plan(starts=ids(5, dtype=ops.DTE_BF16)), "DTE_I32 or DTE_I64")
    refused(plan(tokens=2 ** 24 + 1), "2^24 tokens")
    refused(plan(starts=ids(2 ** 20 + 2)), "2^20 sequences")
    refused(plan(buf=4100), "256-byte aligned")
    refused(plan(buf=None), "null")
    refused(plan(flags=4), "flags")
    need = dte.dte_attention_plan_bytes(1000, 4)
    assert plan(size=need - 1) == 3 and need % 256 == 0
    assert need <= dte.dte_attention_plan_bytes(2000, 4) and need <= dte.dte_attention_plan_bytes(1000, 400)
    # every tile of the sequences, in either size, and the header
    for lengths in ([1] * 4, [997, 1, 1, 1], [250] * 4, [129, 127, 257, 487]):
        tiles = sum(-(-n // 128) + -(-n // 256) for n in lengths)
        assert need >= 256 + 16 * tiles
    assert dte.dte_attention_plan_bytes(2 ** 24 + 1, 1) == dte.dte_attention_plan_bytes(1, 2 ** 20 + 1) == UNFIT
    assert dte.dte_attention_backward_workspace_bytes(2 ** 24 + 1, 1) == dte.dte_attention_backward_workspace_bytes(1, 65536) == UNFIT
    assert dte.dte_attention_backward_workspace_bytes(300, 8) >= 300 * 8 * 4
    # beside delta never more than the sums of all parts
    assert dte.dte_attention_backward_workspace_bytes(2 ** 24, 64) <= 2 ** 24 * 64 * 4 + (75 << 20)
    assert backward(size=dte.dte_attention_backward_workspace_bytes(300, 8) - 1) == 3


def test_gradient_norm_and_clipping_refuse():
    L = dte.lib()
    one = tensor(10) + tensor(0, data=0) + tensor(7, ops.DTE_BF16, 4098)
    total = lambda t=one, n=3, to=4096, ws=4096, size=1 << 20: L.dte_grad_sum_squares(t, n, 0, to, ws, size, -1, None)          # noqa: E731
    clip = lambda t=one, n=3, total=4096, most=1.0, outs=None, norm=4096: L.dte_grad_clip(t, n, total, most, outs, norm, -1, None)   # noqa: E731
    refused(total(), "device")
    refused(clip(), "device")
    refused(clip(outs=one), "device")
    for call in (total, clip):
        refused(call(t=None), "tensors are null")
        refused(call(t=tensor(10, dtype=ops.DTE_I32), n=1), "DTE_F32 or DTE_BF16")
        refused(call(t=tensor(10, data=0), n=1), "data is null")
        refused(call(t=tensor(10, data=4098), n=1), "aligned")
        refused(call(t=tensor(10, ops.DTE_BF16, 4097), n=1), "aligned")
        refused(call(t=tensor(2 ** 44 + 1), n=1), "2^44 elements")
        refused(call(t=tensor(2 ** 43) + tensor(2 ** 43) + tensor(1), n=3), "2^44 elements")
        refused(call(n=2 ** 20 + 1), "2^20 tensors")
    refused(total(to=None), "sum_squares")
    refused(total(to=4100), "sum_squares")
    refused(total(ws=4100), "256-byte aligned")
    assert total(size=100) == 3
    for most in (0.0, -1.0, math.inf, float("nan")):
        refused(clip(most=most), "max_norm")
    refused(clip(total=None), "sum_squares")
    refused(clip(norm=4097), "norm")
    refused(clip(outs=tensor(10) + tensor(0, data=0) + tensor(8, ops.DTE_BF16, 4098)), "sizes")
    refused(clip(t=tensor(10), n=1, outs=tensor(10, ops.DTE_BF16)), "keeps its type")
    sizes = [dte.dte_grad_sum_squares_workspace_bytes(n) for n in (0, 1, 64, 5000, 2 ** 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and all(s % 256 == 0 for s in sizes)
    assert dte.dte_grad_sum_squares_workspace_bytes(2 ** 20 + 1) == UNFIT


def test_the_packed_tensor_has_the_layout_of_the_header():
    assert struct.unpack("=QQII", tensor(5, ops.DTE_BF16, 4096)) == (4096, 5, ops.DTE_BF16, 0)


def test_tensors_off_the_gpu_and_wrong_shapes_are_refused():
    x, t, f = torch.zeros(4, 2, 8), torch.zeros(4, dtype=torch.int64), torch.ones(4, dtype=torch.float64)
    b = torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda: dte.dte_rope(x, None, t, f), lambda: dte.dte_attention_plan(t, 4, b),
                 lambda: dte.dte_attention_forward(x, x, x, b, x, None), lambda: dte.dte_grad_sum_squares([x], f[0], b),
                 lambda: dte.dte_grad_clip([x], f[0], 1.0), lambda: dte.dte_attention_backward(x, x, x, x, x, x, b, x, x, x, b)):
        with pytest.raises(dte.DteError) as e:
            call()
        assert e.value.status == 1
    with pytest.raises(dte.DteError, match="heads x head_dim"):
        ops._heads(x[0], "q", -1)
    with pytest.raises(dte.DteError, match="side by side"):
        ops._heads(x.transpose(0, 1), "q", -1)
    with pytest.raises(dte.DteError, match="side by side"):
        ops._heads(x[..., :4], "q", -1)
    with pytest.raises(dte.DteError, match="float32 or bfloat16"):
        ops._heads(x.half(), "q", -1)
