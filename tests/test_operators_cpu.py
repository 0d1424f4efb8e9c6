"""Host side of the operators, without a GPU: sizes of workspaces, and arguments that are refused before any CUDA call."""
import ctypes

import pytest
import torch

import paper_2608_00455_b200 as dte
from paper_2608_00455_b200 import operators as ops

UNFIT = 2 ** 64 - 1


def matrix(rows, cols, ld=None, dtype=ops.DTE_BF16, data=4096):
    return ops._pack_matrix(data, rows, cols, cols if ld is None else ld, dtype, 0)


def ids(count, dtype=ops.DTE_I64, data=8192):
    return ops._pack_ids(data, count, dtype, 0)


def test_workspace_sizes_grow_with_their_arguments_and_say_when_a_call_would_be_refused():
    for f, args in ((dte.dte_embedding_backward_workspace_bytes, (1000, 512)), (dte.dte_norm_backward_workspace_bytes, (1000, 512)),
                    (dte.dte_linear_ce_forward_workspace_bytes, (1000, 5000, 512)),
                    (dte.dte_linear_ce_backward_workspace_bytes, (1000, 5000, 512)),
                    (dte.dte_linear_ce_backward_workspace_min_bytes, (1000, 5000, 512))):
        base = f(*args)
        assert 0 < base < 2 ** 40 and base % 256 == 0
        for i in range(len(args)):
            more = list(args)
            more[i] *= 4
            assert f(*more) >= base
            more[i] = 2 ** 40
            assert f(*more) == UNFIT
    # logits are not kept: 65536 tokens over 151936 entries would be 20 GB of them in bf16
    assert dte.dte_linear_ce_forward_workspace_bytes(65536, 151936, 4096) < 2 ** 30
    assert dte.dte_linear_ce_backward_workspace_bytes(65536, 151936, 4096) < 2 ** 32
    assert dte.dte_linear_ce_backward_workspace_min_bytes(8192, 151936, 4096) <= dte.dte_linear_ce_backward_workspace_bytes(8192, 151936, 4096)


def refused(status, word):
    assert status == 1
    assert word in dte.lib().dte_last_error().decode()


def test_entry_points_refuse_bad_descriptors_before_any_cuda_call():
    L = dte.lib()
    ok, one = matrix(4, 16), ids(4)
    emb = lambda t, i, o, start=0, vocab=10 ** 6, scale=1.0: L.dte_embedding_forward(t, i, start, vocab, scale, o, None, 0, None)   # noqa: E731
    refused(emb(None, one, ok), "null")
    refused(emb(ok, None, ok), "null")
    refused(emb(matrix(4, 16, dtype=ops.DTE_I32), one, ok), "dtype")
    refused(emb(ok, ids(4, dtype=ops.DTE_F32), ok), "DTE_I32 or DTE_I64")
    refused(emb(matrix(4, 16, data=4097), one, ok), "aligned")
    refused(emb(ok, ids(4, data=8193), ok), "aligned")
    refused(emb(ok, one, matrix(4, 16, ld=15)), "overlap")
    refused(emb(ok, one, matrix(5, 16)), "ids.count x table.cols")
    refused(emb(ok, one, ok, start=7, vocab=10), "inside the vocabulary")
    refused(emb(ok, one, ok, start=2 ** 63, vocab=2 ** 63), "inside the vocabulary")
    refused(emb(ok, one, ok, scale=float("inf")), "finite")
    refused(emb(matrix(2 ** 31, 16), one, ok), "rows < 2^31")
    refused(emb(matrix(4, 0), one, matrix(4, 0)), "cols")
    back = lambda d, i, t, size=1 << 40, ws=4096: L.dte_embedding_backward(d, i, 0, 10 ** 8, 1.0, 0, t, ws, size, None, 0, None)    # noqa: E731
    refused(back(ok, one, matrix(2 ** 21, 16)), "rows of a table")
    refused(back(ok, one, matrix(4, 16), ws=4097), "256-byte aligned")
    assert back(ok, one, matrix(4, 16), size=100) == 3
    norm = lambda x, o, kind=0, eps=1e-6, pdtype=0: L.dte_norm_forward(x, None, None, pdtype, kind, eps, o, None, None, 0, None)     # noqa: E731
    refused(norm(ok, matrix(4, 17)), "shape")
    refused(norm(ok, matrix(4, 16, dtype=ops.DTE_F32)), "type")
    refused(norm(ok, ok, kind=2), "kind")
    refused(norm(ok, ok, eps=float("nan")), "eps")
    refused(norm(ok, ok, pdtype=3), "param_dtype")
    ce = lambda x, w, t, scale=1.0, lse=4096: L.dte_linear_ce_forward(x, w, t, 0, 10 ** 6, scale, lse, None, None, 4096, 1 << 40, None, 0, None)   # noqa: E731
    w = matrix(10, 16)
    refused(ce(matrix(4, 16, dtype=ops.DTE_F32), w, one), "BF16")
    refused(ce(ok, matrix(10, 24), one), "weight.cols")
    refused(ce(matrix(4, 12), matrix(10, 12), one), "multiple of 8")
    refused(ce(ok, matrix(10, 16, ld=20), one), "multiple of 8")
    refused(ce(ok, matrix(10, 16, data=4104), one), "16-byte aligned")
    refused(ce(ok, w, one, scale=-1.0), "logit_scale")
    refused(ce(ok, w, one, lse=None), "lse is null")
    bw = lambda dx, dw, lse=4096: L.dte_linear_ce_backward(ok, w, one, 0, 10 ** 6, 1.0, lse, 4096, 0, dx, dw, 4096, 1 << 40, None, 0, None)   # noqa: E731
    refused(bw(matrix(4, 16), matrix(10, 16), lse=None), "lse / dloss")
    refused(bw(matrix(4, 16, dtype=ops.DTE_F32), None), "dx")
    refused(bw(None, matrix(9, 16)), "weight's shape")
    refused(bw(matrix(4, 16, ld=20), None), "16-byte aligned")


def test_packed_descriptors_have_the_layout_of_the_header():
    class Matrix(ctypes.Structure):
        _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_uint64), ("cols", ctypes.c_uint64), ("ld", ctypes.c_uint64),
                    ("dtype", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]

    class Ids(ctypes.Structure):
        _fields_ = [("data", ctypes.c_void_p), ("count", ctypes.c_uint64), ("dtype", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]

    m = Matrix.from_buffer_copy(matrix(3, 5, 7, ops.DTE_BF16, 4096))
    assert (m.data, m.rows, m.cols, m.ld, m.dtype) == (4096, 3, 5, 7, ops.DTE_BF16)
    i = Ids.from_buffer_copy(ids(9, ops.DTE_I32, 64))
    assert (i.data, i.count, i.dtype) == (64, 9, ops.DTE_I32)


def test_tensors_off_the_gpu_are_refused():
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: dte.dte_embedding_forward(x, t, x), lambda: dte.dte_norm_forward(x, None, None, x, None, None, 1e-6),
                 lambda: dte.dte_linear_ce_forward(x, x, t, x[:, 0], None, None, x), lambda: dte.dte_embedding_forward(None, t, x)):
        with pytest.raises(dte.DteError) as e:
            call()
        assert e.value.status == 1


def test_rows_of_higher_dimensional_tensors():
    t = torch.zeros(3, 4, 8)
    assert ops._rows(t, "t") == (12, 8)
    assert ops._rows(t.expand(3, 4, 8), "t") == (12, 8)
    assert ops._rows(torch.zeros(8), "t") == (1, 8)
    assert ops._rows(torch.zeros(2, 1, 8), "t") == (2, 8)
    assert ops._rows(torch.zeros(2, 5, 16)[..., :8], "t") == (10, 16)
    with pytest.raises(dte.DteError, match="flattened"):
        ops._rows(t[:, :2], "t")


@pytest.mark.parametrize("device", [-1, 64, 2 ** 31 - 1])
def test_every_entry_point_refuses_a_device_ordinal_out_of_range(device):
    L, m, one, w, p, size = dte.lib(), matrix(4, 16), ids(4), matrix(10, 16), 4096, 1 << 40
    for call in (lambda: L.dte_embedding_forward(w, one, 0, 10, 1.0, m, None, device, None),
                 lambda: L.dte_embedding_backward(m, one, 0, 10, 1.0, 0, w, p, size, None, device, None),
                 lambda: L.dte_norm_forward(m, None, None, 0, 0, 1e-6, m, None, None, device, None),
                 lambda: L.dte_norm_backward(m, m, None, 0, 1, None, p, 0, m, None, None, None, 0, device, None),
                 lambda: L.dte_linear_ce_forward(m, w, one, 0, 10, 1.0, p, None, None, p, size, None, device, None),
                 lambda: L.dte_linear_ce_backward(m, w, one, 0, 10, 1.0, p, p, 0, m, w, p, size, None, device, None)):
        refused(call(), "device")


def test_scales_that_fp32_does_not_hold_are_refused():
    # the kernels multiply in fp32: a finite double beyond it would be an infinity there, and 0 * infinity no number
    L, m, one, w, p, size, big = dte.lib(), matrix(4, 16), ids(4), matrix(10, 16), 4096, 1 << 40, 3.5e38
    refused(L.dte_embedding_forward(w, one, 0, 10, big, m, None, -1, None), "scale")
    refused(L.dte_embedding_forward(w, one, 0, 10, -big, m, None, -1, None), "scale")
    refused(L.dte_embedding_backward(m, one, 0, 10, big, 0, w, p, size, None, -1, None), "scale")
    refused(L.dte_norm_forward(m, None, None, 0, 0, big, m, None, None, -1, None), "eps")
    for scale in (big, 2.4e38):                     # the second one is beyond fp32 in base-2 exponents
        refused(L.dte_linear_ce_forward(m, w, one, 0, 10, scale, p, None, None, p, size, None, -1, None), "logit_scale")
        refused(L.dte_linear_ce_backward(m, w, one, 0, 10, scale, p, p, 0, m, w, p, size, None, -1, None), "logit_scale")
    for scale in (3.4e38, -3.4e38):                 # held: only the device is refused
        refused(L.dte_embedding_forward(w, one, 0, 10, scale, m, None, -1, None), "device")
