"""The operators at the two ends of the model - embedding lookup, layer / RMS norm, the linear head's cross
entropy, and their gradients - element by element against their formulas in 64 bits, at the sizes,
strides, masks and types where they can go wrong; gradients against differences as well.

Every tolerance is an element-wise bound made from the operator's own rounding steps: U is the rounding of the
output type, 2^-24 one fp32 rounding, and the factors in front count the longest chain of fp32 operations.
"""
import math

import pytest
import torch

import paper_2608_00455_b200 as dte
from paper_2608_00455_b200 import operators as ops

pytestmark = pytest.mark.gpu

F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
E = 2.0 ** -24
DEV = "cuda"


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def normal(seed, shape, std=1.0, dtype=F32, mean=0.0):
    return torch.empty(shape, dtype=F32, device=DEV).normal_(mean, std, generator=gen(seed)).to(dtype)


def randint(seed, lo, hi, n, dtype=torch.int64):
    return torch.randint(lo, hi, (n,), generator=gen(seed), device=DEV, dtype=dtype)


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


def strided(t, ld, offset):
    """t's values as rows `ld` elements apart, starting `offset` elements into an allocation."""
    buf = torch.zeros(offset + max(1, t.shape[0]) * ld, dtype=t.dtype, device=DEV)
    v = buf[offset:offset + t.shape[0] * ld].view(t.shape[0], ld)[:, :t.shape[1]]
    v.copy_(t)
    return v


# ---- embedding ---------------------------------------------------------------------------------------------

def lookup_case(n, hidden, rows, row_start, seed, id_dtype=torch.int64):
    ids = randint(seed, 0, row_start + rows + 7, n, id_dtype)
    if n > 3:
        ids[1] = -1
        ids[2] = -(2 ** 31)
        ids[n - 1] = row_start + rows - 1
        ids[0] = row_start
    return ids


def local_rows(ids, row_start, rows):
    i = ids.to(torch.int64)
    return torch.where((i >= row_start) & (i < row_start + rows), i - row_start, -1)


@pytest.mark.parametrize("n,hidden,rows", [(1, 8, 1), (2, 1, 3), (33, 100, 50), (257, 1024, 300), (64, 1032, 1000), (5, 4096, 20), (300, 37, 9)])
@pytest.mark.parametrize("table_dtype", [F32, BF16])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_lookup(n, hidden, rows, table_dtype, out_dtype):
    for row_start, id_dtype, extra, offset in ((0, torch.int64, 0, 0), (11, torch.int32, 8, 8), (3, torch.int64, 3, 1)):
        table = strided(normal(1, (rows, hidden), 1.0, table_dtype), hidden + extra, offset)
        ids = lookup_case(n, hidden, rows, row_start, 2, id_dtype)
        out = strided(torch.full((n, hidden), 7.0, dtype=out_dtype, device=DEV), hidden + extra, offset)
        dte.dte_embedding_forward(table, ids, out, scale=1.7, row_start=row_start, vocab=row_start + rows + 7)
        row = local_rows(ids, row_start, rows)
        scale = torch.tensor(1.7, dtype=F32).to(F64).item()
        want = table.to(F64)[row.clamp(min=0)] * scale * (row >= 0)[:, None]
        assert_within(out, want, (U[out_dtype] + 2 * E) * want.abs() + 1e-38, f"out {row_start}")
        assert bool((out[row < 0] == 0).all())


def test_lookup_with_unit_scale_copies_bits_and_other_rows_may_hold_anything():
    table = normal(3, (50, 64), 1.0, BF16)
    table[7] = float("nan")
    table[8] = float("inf")
    ids = torch.tensor([-5, 3, 9, -1, 120, 49], device=DEV)
    out = torch.full((6, 64), float("nan"), dtype=BF16, device=DEV)
    dte.dte_embedding_forward(table, ids, out, vocab=200)
    want = torch.zeros(6, 64, dtype=BF16, device=DEV)
    want[1], want[2], want[5] = table[3], table[9], table[49]
    assert torch.equal(out, want)


def test_lookup_shapes_and_broadcast_table_rows():
    ids = randint(4, 0, 5, 12, torch.int32).view(3, 4)
    row = normal(5, (1, 32))
    table = row.expand(5, 32)                       # stride 0: one row for every id
    out = torch.empty(3, 4, 32, device=DEV)
    dte.dte_embedding_forward(table, ids, out, scale=2.0)
    assert torch.equal(out, (row * 2).expand(12, 32).view(3, 4, 32))
    empty = torch.empty(0, 32, device=DEV)
    dte.dte_embedding_forward(table, ids.view(-1)[:0], empty)


@pytest.mark.parametrize("n,rows,hidden", [(0, 9, 16), (1, 1, 8), (2, 1, 264), (31, 4, 100), (32, 700, 8), (33, 2, 256), (1000, 513, 40),
                                           (5000, 150000, 16), (40000, 3000, 8), (4097, 1, 72), (700, 40, 33)])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
def test_lookup_gradient(n, rows, hidden, types):
    src, dst = types
    for row_start, accumulate, extra, offset in ((0, False, 0, 0), (5, True, 8, 0), (2, False, 3, 1)):
        ids = lookup_case(n, hidden, rows, row_start, 6, torch.int32 if accumulate else torch.int64)
        if n > 200:
            ids[n // 3: n // 3 + n // 5] = row_start + rows // 2       # a token far more frequent than the others
        dout = strided(normal(7, (n, hidden), 1.0, src), hidden + extra, offset)
        row = local_rows(ids, row_start, rows)
        dout[row < 0] = float("nan")                                   # rows of padding and of other shards are not read
        start = normal(8, (rows, hidden), 1.0, dst)
        grad = strided(start, hidden + extra, offset)
        ws = workspace(dte.dte_embedding_backward_workspace_bytes(n, hidden))
        dte.dte_embedding_backward(dout, ids, grad, ws, scale=1.3, row_start=row_start, vocab=row_start + rows + 7, accumulate=accumulate)
        mine = row >= 0
        scale = torch.tensor(1.3, dtype=F32).to(F64).item()
        d = dout[mine].to(F64)
        want = torch.zeros(rows, hidden, dtype=F64, device=DEV).index_add_(0, row[mine], d) * scale
        mass = torch.zeros(rows, hidden, dtype=F64, device=DEV).index_add_(0, row[mine], d.abs()) * scale
        if accumulate:
            want, mass = want + start.to(F64), mass + start.to(F64).abs()
        longest = int(torch.bincount(row[mine], minlength=1).max()) if bool(mine.any()) else 0
        chain = 32 + longest / 32 + 4
        assert_within(grad, want, chain * E * mass + U[dst] * want.abs() * 1.01, f"gradient {row_start} {accumulate}")


def test_lookup_gradient_is_the_adjoint_and_the_same_bits_every_time():
    n, rows, hidden = 3000, 900, 96
    ids = randint(9, 0, rows, n)
    ids[:800] = 17
    dout, table = normal(10, (n, hidden)), normal(11, (rows, hidden))
    out, grads = torch.empty(n, hidden, device=DEV), []
    dte.dte_embedding_forward(table, ids, out, scale=0.5)
    for _ in range(3):
        g = torch.empty(rows, hidden, device=DEV)
        dte.dte_embedding_backward(dout, ids, g, workspace(dte.dte_embedding_backward_workspace_bytes(n, hidden)), scale=0.5)
        grads.append(g)
    assert torch.equal(grads[0], grads[1]) and torch.equal(grads[0], grads[2])
    a = (dout.to(F64) * out.to(F64)).sum().item()
    b = (grads[0].to(F64) * table.to(F64)).sum().item()
    size = (dout.to(F64) * out.to(F64)).abs().sum().item()
    assert abs(a - b) <= 64 * E * size


def test_lookup_flags_ids_past_the_vocabulary():
    table, out = normal(1, (10, 8)), torch.empty(3, 8, device=DEV)
    flags = torch.zeros(1, dtype=torch.int64, device=DEV)
    ids = torch.tensor([1, 9, 14], device=DEV)
    dte.dte_embedding_forward(table, ids, out, vocab=15, flags=flags)
    ws = workspace(dte.dte_embedding_backward_workspace_bytes(3, 8))
    dte.dte_embedding_backward(out, ids, torch.empty_like(table), ws, vocab=15, flags=flags)
    assert flags.item() == 0
    dte.dte_embedding_forward(table, ids, out, vocab=14, flags=flags)
    assert flags.item() == dte.DTE_DEV_BOUNDS and bool((out[2] == 0).all())
    flags.zero_()
    dte.dte_embedding_backward(out, ids, torch.empty_like(table), ws, vocab=14, flags=flags)
    assert flags.item() == dte.DTE_DEV_BOUNDS


# ---- norm -----------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (3, 7), (1, 64), (17, 65), (300, 128), (33, 200), (1000, 256), (5, 257), (2, 1000), (700, 2048), (4, 4096), (3, 4100),
              (3, 5001), (2, 8192), (3, 8200), (5, 20000)]


def norm_inputs(rows, cols, dtype, seed, extra, offset):
    x = normal(seed, (rows, cols), 1.3, F32, 0.7)
    if rows > 2:
        x[1] = 5.0                                   # no variance: rstd is 1 / sqrt(eps)
    return strided(x.to(dtype), cols + extra, offset)


def norm_reference(x, w, b, eps, rms):
    x = x.to(F64)
    mean = torch.zeros(x.shape[0], 1, dtype=F64, device=DEV) if rms else x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    return (x - mean) * rstd * w + b, mean, rstd


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rms", [False, True])
def test_norm_forward_and_backward(rows, cols, dtype, rms):
    eps = torch.tensor(1e-5, dtype=F32).item()
    k = 48 + cols / 256                              # longest chain: a thread's share, the tree, a few products
    for extra, offset, pdtype in ((0, 0, F32), (8, 8, BF16), (3, 1, F32)):
        x = norm_inputs(rows, cols, dtype, 20, extra, offset)
        w, b = normal(21, (cols,), 0.3, pdtype, 1.0), normal(22, (cols,), 0.3, pdtype)
        out = strided(torch.zeros(rows, cols, dtype=dtype, device=DEV), cols + extra, offset)
        mean, rstd = torch.full((rows,), 9.0, device=DEV), torch.empty(rows, device=DEV)
        dte.dte_norm_forward(x, w, b, out, None if rms else mean, rstd, eps, rms=rms)
        w64, b64 = w.to(F64), b.to(F64)
        want, mean64, rstd64 = norm_reference(x, w64, b64, eps, rms)
        size = x.to(F64).abs().mean(1, keepdim=True) * (0 if rms else 1)
        # a shift of the mean by k E size changes rstd by the same in the units of x, and so y twice
        spread = (x.to(F64).abs() + 2 * size) * rstd64
        spread = spread * (1 + size * rstd64)
        assert_within(out, want, U[dtype] * want.abs() * 1.01 + k * E * (w64.abs() * spread + b64.abs()), "out")
        if not rms:
            assert_within(mean, mean64[:, 0], k * E * size[:, 0], "mean")
        rel = k * E * (1 + (size * rstd64) ** 2)
        assert_within(rstd, rstd64[:, 0], (rel * rstd64)[:, 0], "rstd")

        dout = strided(normal(23, (rows, cols), 1.0, dtype), cols + extra, offset)
        dx = strided(torch.zeros(rows, cols, dtype=dtype, device=DEV), cols + extra, offset)
        dw0, db0 = normal(24, (cols,)), normal(25, (cols,))
        for accumulate in (False, True):
            dw, db = dw0.clone(), db0.clone()
            ws = workspace(dte.dte_norm_backward_workspace_bytes(rows, cols))
            dte.dte_norm_backward(dout, x, w, None if rms else mean, rstd, dx, dw, db, ws, accumulate=accumulate, rms=rms)
            # the formula at the statistics that were passed
            m, r = (torch.zeros_like(rstd) if rms else mean).to(F64)[:, None], rstd.to(F64)[:, None]
            xh, ax = (x.to(F64) - m) * r, (x.to(F64).abs() + m.abs()) * r
            dy = dout.to(F64)
            g = dy * w64
            c2 = (g * xh).mean(1, keepdim=True)
            wdx = r * (g - (0 if rms else g.mean(1, keepdim=True)) - xh * c2)
            mag = r * (g.abs() + g.abs().mean(1, keepdim=True) + ax * (g.abs() * ax).mean(1, keepdim=True))
            assert_within(dx, wdx, U[dtype] * wdx.abs() * 1.01 + k * E * mag, "dx")
            chain = 40 + rows / 64
            wdw, wdb = (dy * xh).sum(0), dy.sum(0)
            mdw, mdb = (dy.abs() * ax).sum(0), dy.abs().sum(0)
            if accumulate:
                wdw, wdb, mdw, mdb = wdw + dw0, wdb + db0, mdw + dw0.abs(), mdb + db0.abs()
            assert_within(dw, wdw, chain * E * mdw, "dweight")
            assert_within(db, wdb, chain * E * mdb, "dbias")


@pytest.mark.parametrize("rows,cols", [(3, 7), (17, 65), (300, 128), (33, 200), (5, 257), (700, 2048), (40, 4096), (6, 4100), (5, 8192), (4, 8200), (3, 20000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm_gradient_of_rows_with_an_offset(rows, cols, dtype):
    # rows whose mean is far larger than their deviation, and rows without any: xhat is as exact as x - mean is
    eps = torch.tensor(1e-5, dtype=F32).item()
    k = 48 + cols / 256
    for extra, offset in ((0, 0), (3, 1)):
        x = normal(140, (rows, cols))
        x[0] += 1000.0
        x[1] = -5.0
        x[2] = x[2] * 1e-2 + 300.0
        x[rows // 2] += -1e4
        x = strided(x.to(dtype), cols + extra, offset)
        w = normal(141, (cols,), 0.3, F32, 1.0)
        _, m, r = norm_reference(x, w.to(F64), 0.0, eps, False)
        mean, rstd = m[:, 0].to(F32), r[:, 0].to(F32)
        dout = strided(normal(142, (rows, cols), 1.0, dtype), cols + extra, offset)
        dx = strided(torch.zeros(rows, cols, dtype=dtype, device=DEV), cols + extra, offset)
        dw, db = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
        dte.dte_norm_backward(dout, x, w, mean, rstd, dx, dw, db, workspace(dte.dte_norm_backward_workspace_bytes(rows, cols)))
        # the formula at the statistics that were passed; x - mean is rounded once, so all is relative to its size
        m, r = mean.to(F64)[:, None], rstd.to(F64)[:, None]
        xh, dy = (x.to(F64) - m) * r, dout.to(F64)
        g = dy * w.to(F64)
        wdx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        mag = r * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
        assert_within(dx, wdx, U[dtype] * wdx.abs() * 1.01 + k * E * mag, "dx")
        chain = 40 + rows / 64
        assert_within(dw, (dy * xh).sum(0), chain * E * (dy * xh).abs().sum(0), "dweight")
        assert_within(db, dy.sum(0), chain * E * dy.abs().sum(0), "dbias")


def test_norm_optional_parts():
    x, dy = normal(30, (50, 384), 1.0, BF16), normal(31, (50, 384), 1.0, BF16)
    out, plain = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(50, device=DEV), torch.empty(50, device=DEV)
    one, zero = torch.ones(384, device=DEV), torch.zeros(384, device=DEV)
    dte.dte_norm_forward(x, one, zero, out, mean, rstd, 1e-6)
    dte.dte_norm_forward(x, None, None, plain, None, None, 1e-6)          # no weights, no statistics kept
    assert torch.equal(out, plain)
    ws = workspace(dte.dte_norm_backward_workspace_bytes(50, 384))
    dx, dw, db = torch.empty_like(x), torch.empty(384, device=DEV), torch.empty(384, device=DEV)
    dte.dte_norm_backward(dy, x, one, mean, rstd, dx, dw, db, ws)
    dx2, dw2, db2 = torch.empty_like(x), torch.empty(384, device=DEV), torch.empty(384, device=DEV)
    dte.dte_norm_backward(dy, x, None, mean, rstd, dx2, None, None, None)
    dte.dte_norm_backward(dy, x, None, mean, rstd, None, dw2, None, ws)
    dte.dte_norm_backward(dy, x, None, mean, rstd, None, None, db2, ws)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_norm_without_rows():
    x, dw = torch.empty(0, 64, device=DEV), torch.full((64,), 3.0, device=DEV)
    s = torch.empty(0, device=DEV)
    dte.dte_norm_forward(x, None, None, torch.empty_like(x), s, s, 1e-6)
    ws = workspace(dte.dte_norm_backward_workspace_bytes(0, 64))
    dte.dte_norm_backward(x, x, None, s, s, None, dw, None, ws, accumulate=True)
    assert bool((dw == 3).all())
    dte.dte_norm_backward(x, x, None, s, s, None, dw, None, ws)
    assert bool((dw == 0).all())


def test_norm_with_a_broadcast_gradient_and_higher_shapes():
    x = normal(32, (4, 6, 128), 1.0, F32)
    g = normal(33, (1, 128))
    mean, rstd, out = torch.empty(24, device=DEV), torch.empty(24, device=DEV), torch.empty_like(x)
    dte.dte_norm_forward(x, None, None, out, mean, rstd, 1e-6)
    dx, full = torch.empty_like(x), torch.empty_like(x)
    dw, dw2 = torch.empty(128, device=DEV), torch.empty(128, device=DEV)
    ws = workspace(dte.dte_norm_backward_workspace_bytes(24, 128))
    dte.dte_norm_backward(g.expand(24, 128), x, None, mean, rstd, dx, dw, None, ws)       # row stride 0
    dte.dte_norm_backward(g.expand(24, 128).contiguous(), x, None, mean, rstd, full, dw2, None, ws)
    assert torch.equal(dx, full) and torch.equal(dw, dw2)


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradient_against_differences(rms):
    rows, cols, h = 6, 264, 2.0 ** -7
    x, w, b, c = normal(34, (rows, cols)), normal(35, (cols,), 0.3, F32, 1.0), normal(36, (cols,)), normal(37, (rows, cols))

    def value(x, w, b):
        out = torch.empty_like(x)
        dte.dte_norm_forward(x, w, b, out, None, None, 1e-6, rms=rms)
        return (out.to(F64) * c.to(F64)).sum().item()

    out, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    dte.dte_norm_forward(x, w, b, out, None if rms else mean, rstd, 1e-6, rms=rms)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    dte.dte_norm_backward(c, x, w, None if rms else mean, rstd, dx, dw, db, workspace(dte.dte_norm_backward_workspace_bytes(rows, cols)), rms=rms)
    # along the sign of each gradient: the derivative is its 1-norm; the central difference is off by O(h^2)
    # relative, and by the rounding of the sum (64 E of its terms) over 2 h
    noise = 64 * E * (out.abs() * c.abs()).sum().item() / (2 * h)
    for g, at in ((dx, lambda s: value(x + s, w, b)), (dw, lambda s: value(x, w + s, b)), (db, lambda s: value(x, w, b + s))):
        d = g.sign() * h
        slope = g.abs().to(F64).sum().item()
        assert abs((at(d) - at(-d)) / (2 * h) - slope) <= 0.01 * slope + noise


# ---- cross entropy of a linear head ------------------------------------------------------------------------

def head_case(tokens, vocab, hidden, seed, ignored=0.0, start=0, total=None):
    x = normal(seed, (tokens, hidden), 1.0, BF16)
    w = normal(seed + 1, (vocab, hidden), 2.0 / math.sqrt(hidden), BF16)
    t = randint(seed + 2, 0, total or vocab, tokens)
    if ignored:
        t[torch.rand(tokens, generator=gen(seed + 3), device=DEV) < ignored] = -100
    return x, w, t


class Head:
    """The formulas in 64 bits, with element-wise error bounds."""

    def __init__(self, x, w, t, scale=1.0, start=0):
        self.t, self.scale, self.start = t, scale, start
        self.keep = t >= 0
        self.x = torch.where(self.keep[:, None], x, 0).to(F64)
        self.w = w.to(F64)
        self.z = scale * self.x @ self.w.T
        hidden = x.shape[1]
        # a product of `hidden` terms adds up 16 at a time in fp32, possibly truncated: 2^-23 per step
        self.dz = (hidden / 16 + 16) * 2.0 ** -23 * scale * (self.x.abs() @ self.w.abs().T)
        col = t - start
        self.here = self.keep & (col >= 0) & (col < w.shape[0])
        self.col = torch.where(self.here, col, 0)
        self.lse = torch.where(self.keep, torch.logsumexp(self.z, 1), 0.0)
        self.tl = torch.where(self.here, self.z.gather(1, self.col[:, None])[:, 0], 0.0)
        self.dtl = torch.where(self.here, self.dz.gather(1, self.col[:, None])[:, 0], 0.0)
        # statistics: a shift of the logits shifts the sum; exponentials are good to 2^-21, arguments to 4 E of their size
        self.dlse = torch.where(self.keep, self.dz.amax(1) + 2.0 ** -20 + 8 * E * (self.lse.abs() + self.z.abs().amax(1)), 0.0)

    def check_forward(self, lse, tl, loss):
        assert_within(lse, self.lse, self.dlse, "lse")
        assert_within(tl, self.tl, self.dtl + 2 * E * self.tl.abs(), "target_logit")
        assert_within(loss, torch.where(self.keep, self.lse - self.tl, 0.0),
                      self.dlse + self.dtl + 4 * E * (self.lse.abs() + self.tl.abs()), "loss")
        for v in (lse, tl, loss):
            assert bool((v[~self.keep] == 0).all())

    def gradients(self, dloss, lse, kept=2.0 ** -8):
        """(dx, bound, dw, bound) for fp32 lse as passed; kept: how closely f p is kept (bf16: 8 significant bits)."""
        f = torch.where(self.keep, dloss.to(F64), 0.0) * self.scale
        p = torch.exp(self.z - lse.to(F64)[:, None]) * self.keep[:, None]
        g = f[:, None] * p
        # p as it is kept, from exponents that are off by dz and by fp32 roundings of their size
        rel = kept + 1.1 * (self.dz + 8 * E * (self.z.abs() + lse.to(F64).abs()[:, None]) + 2.0 ** -20)
        dg = g.abs() * rel
        hot = torch.zeros_like(g)
        hot[torch.arange(len(f), device=DEV), self.col] = f * self.here
        n, v = g.shape
        dx, dw = (g - hot) @ self.w, (g - hot).T @ self.x
        mx, mw = (g.abs() + hot.abs()) @ self.w.abs(), (g.abs() + hot.abs()).T @ self.x.abs()
        # fp32 sums over the vocabulary and over the tokens: 16 at a time on the tensor cores, truncated
        bx = dg @ self.w.abs() + (v / 16 + 64) * 2.0 ** -23 * mx
        bw = dg.T @ self.x.abs() + (n / 16 + 64) * 2.0 ** -23 * mw
        return dx, bx, dw, bw


def run_forward(x, w, t, scale=1.0, start=0, total=None, flags=None):
    n = t.numel()
    lse, tl, loss = (torch.full((n,), float("nan"), device=DEV) for _ in range(3))
    ws = workspace(dte.dte_linear_ce_forward_workspace_bytes(n, w.shape[0], w.shape[1]))
    dte.dte_linear_ce_forward(x, w, t, lse, tl, loss, ws, logit_scale=scale, vocab_start=start, vocab=total, flags=flags)
    return lse, tl, loss


def run_backward(x, w, t, lse, dloss, scale=1.0, start=0, total=None, dw=None, accumulate=False, small=False, dx=None):
    n, v, h = t.numel(), w.shape[0], w.shape[1]
    dx = torch.full((n, h), float("nan"), dtype=BF16, device=DEV) if dx is None else dx
    dw = torch.full((v, h), float("nan"), dtype=BF16, device=DEV) if dw is None else dw
    size = dte.dte_linear_ce_backward_workspace_min_bytes if small else dte.dte_linear_ce_backward_workspace_bytes
    flags = torch.zeros(1, dtype=torch.int64, device=DEV)
    dte.dte_linear_ce_backward(x, w, t, lse, dloss, dx, dw, workspace(size(n, v, h)), logit_scale=scale, vocab_start=start, vocab=total,
                               accumulate=accumulate, flags=flags)
    assert flags.item() == 0
    return dx, dw


HEAD_SIZES = [(1, 1, 8), (1, 256, 64), (2, 5, 72), (8, 3000, 128), (127, 257, 64), (128, 255, 320), (129, 256, 8), (255, 700, 200),
              (256, 513, 256), (257, 300, 264), (300, 2049, 512), (700, 1000, 1032), (3, 20000, 2048)]


@pytest.mark.parametrize("tokens,vocab,hidden", HEAD_SIZES)
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_head_forward(tokens, vocab, hidden, ignored):
    x, w, t = head_case(tokens, vocab, hidden, 40, ignored)
    flags = torch.zeros(1, dtype=torch.int64, device=DEV)
    got = run_forward(x, w, t, flags=flags)
    assert flags.item() == 0
    Head(x, w, t).check_forward(*got)


@pytest.mark.parametrize("tokens,vocab,hidden", HEAD_SIZES)
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_head_gradients(tokens, vocab, hidden, ignored):
    x, w, t = head_case(tokens, vocab, hidden, 50, ignored)
    ref = Head(x, w, t)
    lse, dloss = ref.lse.to(F32), normal(54, (tokens,))
    dx, dw = run_backward(x, w, t, lse, dloss)
    wx, bx, ww, bw = ref.gradients(dloss, lse)
    assert_within(dx, wx, bx + U[BF16] * wx.abs() * 1.01, "dx")
    assert_within(dw, ww, bw + U[BF16] * ww.abs() * 1.01, "dweight")
    assert bool((dx[~ref.keep] == 0).all())


def test_head_many_tiles_and_pieces():
    # more tiles than SMs in every product, several pieces of the vocabulary with a ragged last one
    tokens, vocab, hidden = 1500, 9001, 1288
    x, w, t = head_case(tokens, vocab, hidden, 60, 0.2)
    ref = Head(x, w, t, scale=0.8)
    got = run_forward(x, w, t, scale=0.8)
    ref.check_forward(*got)
    lse, dloss = got[0], normal(61, (tokens,))
    wx, bx, ww, bw = ref.gradients(dloss, lse)
    for small in (False, True):
        dx, dw = run_backward(x, w, t, lse, dloss, scale=0.8, small=small)
        assert_within(dx, wx, bx + U[BF16] * wx.abs() * 1.01, "dx")
        assert_within(dw, ww, bw + U[BF16] * ww.abs() * 1.01, "dweight")


@pytest.mark.parametrize("tokens,vocab,hidden", [(1998, 18844, 2040), (9400, 700, 1016)])
def test_head_many_rounds_of_tiles(tokens, vocab, hidden):
    # whole rounds of tiles over 148 SMs, with ragged edges: in the logits and dweight, and in dx
    x, w, t = head_case(tokens, vocab, hidden, 80, 0.01)
    ref = Head(x, w, t)
    got = run_forward(x, w, t)
    ref.check_forward(*got)
    lse, dloss = got[0], normal(81, (tokens,))
    wx, bx, ww, bw = ref.gradients(dloss, lse)
    dx, dw = run_backward(x, w, t, lse, dloss)
    assert_within(dx, wx, bx + U[BF16] * wx.abs() * 1.01, "dx")
    assert_within(dw, ww, bw + U[BF16] * ww.abs() * 1.01, "dweight")


@pytest.mark.parametrize("tokens,vocab,hidden,ignored", [(1, 700, 64, 0.0), (5, 3000, 200, 0.0), (64, 1000, 264, 0.0), (64, 5000, 128, 0.5),
                                                         (33, 9000, 1032, 0.2)])
def test_head_gradients_of_few_tokens_are_closer_than_bf16(tokens, vocab, hidden, ignored):
    # f p as two bf16 numbers: 2^-17 of it is lost at most; an fp32 weight gradient shows it
    x, w, t = head_case(tokens, vocab, hidden, 100, ignored)
    for start, total in ((0, vocab), (vocab, 2 * vocab)):            # with the targets in the shard, and with none of them
        ref = Head(x, w, t, start=start)
        lse, dloss = ref.lse.to(F32), normal(101, (tokens,))
        wx, bx, ww, bw = ref.gradients(dloss, lse, kept=2.0 ** -16)
        for small in (False, True):
            dw = torch.full((vocab, hidden), float("nan"), device=DEV)
            dx, dw = run_backward(x, w, t, lse, dloss, dw=dw, start=start, total=total, small=small)
            assert_within(dw, ww, bw + 4 * E * ww.abs(), "dweight")
            assert_within(dx, wx, bx + U[BF16] * wx.abs() * 1.01, "dx")
            assert bool((dx[~ref.keep] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_head_accumulates_into_a_gradient_of_either_type(dtype):
    tokens, vocab, hidden = 200, 900, 136
    x, w, t = head_case(tokens, vocab, hidden, 62)
    ref = Head(x, w, t)
    lse, dloss, start = ref.lse.to(F32), normal(63, (tokens,)), normal(64, (vocab, hidden), 1.0, dtype)
    _, _, ww, bw = ref.gradients(dloss, lse)
    for accumulate in (False, True):
        dw = strided(start, hidden + 8, 8)
        run_backward(x, w, t, lse, dloss, dw=dw, accumulate=accumulate)
        want = ww + start.to(F64) if accumulate else ww
        assert_within(dw, want, bw + U[dtype] * want.abs() * 1.01 + 2 * E * ww.abs(), "dweight")


def test_head_on_vocabulary_shards_adds_up_to_the_whole():
    tokens, vocab, hidden, parts = 150, 1200, 96, 3
    x, w, t = head_case(tokens, vocab, hidden, 65, 0.2)
    ref = Head(x, w, t)
    rows = vocab // parts
    lses, tls = [], []
    for r in range(parts):
        lse, tl, _ = run_forward(x, w[r * rows:(r + 1) * rows], t, start=r * rows, total=vocab)
        lses.append(lse.to(F64))
        tls.append(tl.to(F64))
    lse = torch.where(ref.keep, torch.logsumexp(torch.stack(lses), 0), 0.0)
    assert_within(lse, ref.lse, ref.dlse, "lse")
    assert_within(sum(tls), ref.tl, ref.dtl + 2 * E * ref.tl.abs(), "target_logit")
    dloss, lse = normal(66, (tokens,)), lse.to(F32)
    wx, bx, ww, bw = ref.gradients(dloss, lse)
    total, slack = torch.zeros(tokens, hidden, dtype=F64, device=DEV), 0
    for r in range(parts):
        dx, dw = run_backward(x, w[r * rows:(r + 1) * rows], t, lse, dloss, start=r * rows, total=vocab)
        part = slice(r * rows, (r + 1) * rows)
        assert_within(dw, ww[part], bw[part] + U[BF16] * ww[part].abs() * 1.01, "dweight")
        total += dx.to(F64)
        slack = slack + U[BF16] * dx.to(F64).abs() * 1.01
    assert_within(total, wx, bx + slack, "dx")


def test_head_ignored_rows_are_never_read_and_all_ignored_is_zero():
    tokens, vocab, hidden = 140, 600, 128
    x, w, t = head_case(tokens, vocab, hidden, 67, 0.5)
    dirty = x.clone()
    dirty[t < 0] = float("nan")
    dirty[int((t < 0).nonzero()[0])] = float("inf")
    dloss = normal(68, (tokens,))
    dirty_dloss = torch.where(t < 0, float("nan"), dloss)
    a, b = run_forward(x, w, t), run_forward(dirty, w, t)
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    for u, v in zip(run_backward(x, w, t, a[0], dloss), run_backward(dirty, w, t, b[0], dirty_dloss)):
        assert torch.equal(u, v) and bool(torch.isfinite(u.float()).all())
    t.fill_(-1)
    for v in run_forward(dirty, w, t):
        assert bool((v == 0).all())
    for v in run_backward(dirty, w, t, a[0], dloss):
        assert bool((v == 0).all())
    keep = normal(69, (vocab, hidden), 1.0, BF16)
    dw = keep.clone()
    run_backward(dirty, w, t, a[0], dloss, dw=dw, accumulate=True)
    assert torch.equal(dw, keep)


def test_head_without_tokens():
    w = normal(70, (40, 16), 1.0, BF16)
    x, t, e = torch.empty(0, 16, dtype=BF16, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    run_forward(x, w, t)
    _, dw = run_backward(x, w, t, e, e)
    assert bool((dw == 0).all())


def test_head_extreme_logits():
    # a row far above all others, a row of -inf weights, and rows that make a whole token -inf
    tokens, vocab, hidden = 4, 300, 64
    x = torch.zeros(tokens, hidden, dtype=BF16, device=DEV)
    x[:, 0] = 1.0
    w = torch.zeros(vocab, hidden, dtype=BF16, device=DEV)
    w[:, 0] = torch.linspace(-3, 3, vocab, device=DEV).to(BF16)
    w[17, 0], w[5, 0] = 3.0e4, -3.0e38
    t = torch.tensor([17, 5, 3, 299], device=DEV)
    lse, tl, loss = run_forward(x, w, t)
    assert bool((lse == w[17, 0].float()).all())
    assert tl[0].item() == w[17, 0].item() and loss[0].item() == 0.0
    assert loss[1].item() > 1e38
    w[:, 0] = float("-inf")
    lse, tl, loss = run_forward(x[:, :].contiguous(), w, t)
    assert bool((lse == float("-inf")).all())


def test_head_strides_types_and_optional_outputs():
    tokens, vocab, hidden = 77, 333, 72
    x, w, t = head_case(tokens, vocab, hidden, 71, 0.3)
    want = run_forward(x, w, t)
    odd = strided(x, hidden + 3, 1)                     # rows of x at any alignment
    wide = strided(w, hidden + 16, 8)
    got = run_forward(odd, wide, t.to(torch.int32))
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    lse = torch.empty(tokens, device=DEV)
    ws = workspace(dte.dte_linear_ce_forward_workspace_bytes(tokens, vocab, hidden))
    dte.dte_linear_ce_forward(x, w, t, lse, None, None, ws)
    assert torch.equal(lse, want[0])
    dloss = normal(72, (tokens,))
    dx, dw = run_backward(x, w, t, lse, dloss)
    dx2 = strided(torch.zeros(tokens, hidden, dtype=BF16, device=DEV), hidden + 24, 16)
    dw2 = strided(torch.zeros(vocab, hidden, dtype=BF16, device=DEV), hidden + 8, 8)
    run_backward(odd, wide, t, lse, dloss, dx=dx2, dw=dw2)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    ws = workspace(dte.dte_linear_ce_backward_workspace_bytes(tokens, vocab, hidden))
    dx3, dw3 = torch.empty_like(dx), torch.empty_like(dw)
    dte.dte_linear_ce_backward(x, w, t, lse, dloss, dx3, None, ws)
    dte.dte_linear_ce_backward(x, w, t, lse, dloss, None, dw3, ws)
    assert torch.equal(dx, dx3) and torch.equal(dw, dw3)
    one = x[:1].expand(tokens, hidden)                  # a broadcast row
    a, b = run_forward(one, w, t), run_forward(one.contiguous(), w, t)
    assert torch.equal(a[0], b[0])


def test_head_gradient_against_differences():
    tokens, vocab, hidden, h = 20, 150, 64, 2.0 ** -6
    # values on a grid of 2^-6 that bf16 holds together with their neighbours one step away
    x = (normal(73, (tokens, hidden), 0.4).clamp(-1.5, 1.5) / h).round() * h
    w = (normal(74, (vocab, hidden), 0.2).clamp(-1.5, 1.5) / h).round() * h
    t, c = randint(75, 0, vocab, tokens), normal(76, (tokens,)).abs() + 0.5
    assert torch.equal((x + h).to(BF16).to(F32), x + h) and torch.equal((w - h).to(BF16).to(F32), w - h)

    def value(x, w):
        loss = run_forward(x.to(BF16), w.to(BF16), t)[2]
        return (loss.to(F64) * c.to(F64)).sum().item()

    lse, _, loss = run_forward(x.to(BF16), w.to(BF16), t)
    dx, dw = run_backward(x.to(BF16), w.to(BF16), t, lse, c)
    # along the signs of a sixteenth of the entries, so that the logits move by less than 0.1: O(h^2) is below 1 %
    noise = 2.0 ** -18 * (loss.abs() * c).sum().item() / (2 * h)
    for g, at in ((dx, lambda s: value(x + s, w)), (dw, lambda s: value(x, w + s))):
        pick = torch.rand(g.shape, generator=gen(77), device=DEV) < 1 / 16
        d = g.float().sign() * pick * h
        slope = (g.to(F64).abs() * pick).sum().item()
        assert abs((at(d) - at(-d)) / (2 * h) - slope) <= 0.02 * slope + noise


def test_head_same_bits_every_time():
    tokens, vocab, hidden = 400, 5000, 256
    x, w, t = head_case(tokens, vocab, hidden, 78, 0.1)
    dloss = normal(79, (tokens,))
    first = None
    for _ in range(3):
        lse, tl, loss = run_forward(x, w, t)
        got = (lse, tl, loss, *run_backward(x, w, t, lse, dloss))
        first = first or got
        for a, b in zip(first, got):
            assert torch.equal(a, b)


# ---- gradients of tokens whose loss is near zero --------------------------------------------------------------------

def confident_case(tokens, vocab, hidden, seed, ignored=0.0, total=None, start=0, scale=1.0):
    """Tokens with losses from about 1 down to 1e-6: x is a multiple of the target's row of w.  All values lie on grids so
    coarse (w: 2^-4, x: 2^-3) that every logit and every partial sum of one is exact in fp32 whatever the order."""
    w = (normal(seed, (vocab, hidden), 2.2 / math.sqrt(hidden)) * 16).round() / 16
    w = torch.where(w == 0, 1 / 16, w)                 # no empty row
    t = randint(seed + 1, 0, total or vocab, tokens)
    if ignored:
        t[torch.rand(tokens, generator=gen(seed + 2), device=DEV) < ignored] = -100
    col = (t - start).clamp(0, vocab - 1)
    # z_t = scale * gain * |w_t|^2 between log(vocab) and log(vocab) + 14
    want = math.log(vocab) + 14 * torch.arange(tokens, device=DEV) / max(1, tokens - 1)
    gain = want / scale / (w[col] ** 2).sum(1)
    x = (gain[:, None] * w[col] * 8).round() / 8
    assert torch.equal(x.to(BF16).float(), x) and torch.equal(w.to(BF16).float(), w)
    assert float((x.abs() @ w.abs().T).max()) < 2 ** (24 - 7)
    return x.to(BF16), w.to(BF16), t


def centred_gradients(ref, dloss, lse, kept=2.0 ** -8, dzt=0.0):
    """(dx, bound, dw, bound) for fp32 lse as passed.  The target's coefficient f (p - 1) is granted fp32 roundings of its
    own size, of the subtraction z - lse, and dzt, the error of its logit; the other columns f p as it is kept."""
    f = torch.where(ref.keep, dloss.to(F64), 0.0) * ref.scale
    lse = lse.to(F64)[:, None]
    g = f[:, None] * torch.exp(ref.z - lse) * ref.keep[:, None]
    dg = g.abs() * (kept + 1.1 * (ref.dz + 8 * E * (ref.z.abs() + lse.abs()) + 2.0 ** -20))
    row = ref.here.nonzero()[:, 0]
    d = (ref.z - lse)[row, ref.col[row]]
    # f: two roundings, expm1f: 2 E, the product and the sum it goes into: 8 E; z - lse rounds to E |z - lse|
    g[row, ref.col[row]] = f[row] * torch.expm1(d)
    dg[row, ref.col[row]] = f[row].abs() * (8 * E * torch.expm1(d).abs() + torch.exp(d) * (2 * E * d.abs() + dzt))
    n, v = g.shape
    bx = dg @ ref.w.abs() + (v / 16 + 64) * 2.0 ** -23 * (g.abs() @ ref.w.abs())
    bw = dg.T @ ref.x.abs() + (n / 16 + 64) * 2.0 ** -23 * (g.abs().T @ ref.x.abs())
    return g @ ref.w, bx, g.T @ ref.x, bw


@pytest.mark.parametrize("tokens,vocab,hidden,ignored", [(7, 700, 64, 0.0), (64, 2049, 512, 0.2), (65, 2049, 512, 0.0), (128, 300, 72, 0.0),
                                                         (300, 2049, 512, 0.0), (921, 5000, 264, 0.3)])
@pytest.mark.parametrize("scale", [1.0, 0.5])
def test_head_gradients_of_confident_tokens(tokens, vocab, hidden, ignored, scale):
    for start, total in ((0, vocab), (vocab // 3, 2 * vocab)):       # the whole vocabulary; a shard without some of the targets
        x, w, t = confident_case(tokens, vocab, hidden, 110, ignored, total, start, scale)
        ref = Head(x, w, t, scale, start)
        lse = ref.lse.to(F32)
        for dloss in (torch.full((tokens,), 1.0 / 921, device=DEV), normal(113, (tokens,))):
            kept = 2.0 ** -16 if tokens <= 64 else 2.0 ** -8
            wx, bx, ww, bw = centred_gradients(ref, dloss, lse, kept)
            for small in (False, True):
                dw = torch.full((vocab, hidden), float("nan"), device=DEV)
                dx, dw = run_backward(x, w, t, lse, dloss, scale=scale, start=start, total=total, dw=dw, small=small)
                assert_within(dw, ww, bw + 4 * E * ww.abs(), "dweight")
                assert_within(dx, wx, bx + U[BF16] * wx.abs() * 1.01, "dx")
        # what is granted says something: a few per cent at most of the gradient of any token that has a target here
        if tokens > 64:
            part = (bx.norm(dim=1) / wx.norm(dim=1))[ref.here]
            assert float(part.max()) < 0.1


@pytest.mark.parametrize("tokens", [40, 300])
def test_head_gradients_of_confident_tokens_off_the_grid(tokens):
    vocab, hidden = 3000, 1288
    x, w, t = confident_case(tokens, vocab, hidden, 120, scale=0.75)
    x = (x.float() * (1 + normal(123, x.shape, 0.01))).to(BF16)
    ref = Head(x, w, t, 0.75)
    lse, _, loss = run_forward(x, w, t, scale=0.75)
    dloss = normal(124, (tokens,))
    # the logit's sum in fp32: hidden / 256 terms of 8 columns per thread, 16 further additions, one product
    dzt = ((hidden / 256 + 24) * E * 0.75 * (ref.x.abs() @ ref.w.abs().T))[torch.arange(tokens, device=DEV), ref.col]
    wx, bx, ww, bw = centred_gradients(ref, dloss, lse, dzt=dzt)
    dx, dw = run_backward(x, w, t, lse, dloss, scale=0.75, dw=torch.full((vocab, hidden), float("nan"), device=DEV))
    assert_within(dx, wx, bx + U[BF16] * wx.abs() * 1.01, "dx")
    assert_within(dw, ww, bw + 4 * E * ww.abs(), "dweight")


def test_head_training_on_what_is_known_leaves_weights_alone():
    # the gradient of a mean loss over tokens that are all but certain, against that of the same tokens with their targets
    # exchanged: a spurious 2^-9 of f in the target's column would be 1e-3 of it
    tokens, vocab, hidden = 256, 1024, 256
    x, w, t = confident_case(tokens, vocab, hidden, 130)
    x = torch.cat([x[-64:]] * 4)
    t = t[-64:].repeat(4)
    lse, _, loss = run_forward(x, w, t)
    assert float(loss.max()) < 1e-3
    dloss = torch.full((tokens,), 1.0 / 921, device=DEV)
    known, _ = run_backward(x, w, t, lse, dloss)
    other, _ = run_backward(x, w, (t + 1) % vocab, lse, dloss)
    # |dx| = f |sum p (w_v - w_t)| <= f (1 - p) * 2 max |w|, and p = exp(-loss)
    limit = dloss * (loss + 32 * E * lse.abs()) * 2 * w.float().norm(dim=1).max()
    assert bool((known.float().norm(dim=1) <= limit * 1.02).all())
    assert bool((other.float().norm(dim=1) > 1e3 * known.float().norm(dim=1)).all())


@pytest.mark.parametrize("tokens,vocab,hidden", [(4, 300, 64), (300, 700, 64), (40, 60000, 64), (300, 60000, 64), (300, 3000, 1032)])
def test_head_waits_that_run_out_are_reported_and_the_next_call_is_right(tokens, vocab, hidden):
    # one CTA and pairs, one tile and several per CTA, more steps along K than stages: loads are in flight when the waits give up
    x, w, t = head_case(tokens, vocab, hidden, 170)
    dloss = normal(173, (tokens,))
    lse, tl, loss = run_forward(x, w, t)
    want = (lse, tl, loss, *run_backward(x, w, t, lse, dloss))
    flags = torch.zeros(1, dtype=torch.int64, device=DEV)
    ws = workspace(max(dte.dte_linear_ce_forward_workspace_bytes(tokens, vocab, hidden),
                       dte.dte_linear_ce_backward_workspace_bytes(tokens, vocab, hidden)))
    spare, dx, dw = torch.empty_like(lse), torch.empty_like(x), torch.empty_like(w)
    dte.lib().dte_linear_ce_set_wait_limit(1)
    try:
        dte.dte_linear_ce_forward(x, w, t, spare, None, None, ws, flags=flags)
        assert flags.item() == dte.DTE_DEV_TIMEOUT
        flags.zero_()
        dte.dte_linear_ce_backward(x, w, t, lse, dloss, dx, dw, ws, flags=flags)
        assert flags.item() == dte.DTE_DEV_TIMEOUT
    finally:
        dte.lib().dte_linear_ce_set_wait_limit(0)
    flags.zero_()
    got = run_forward(x, w, t, flags=flags)
    for a, b in zip(want, (*got, *run_backward(x, w, t, lse, dloss))):
        assert torch.equal(a, b)
    assert flags.item() == 0


# ---- offsets beyond 32 bits ------------------------------------------------------------------------------------

def test_lookup_and_its_gradient_in_a_table_of_more_than_2_to_the_32_bytes_and_elements():
    rows, hidden, n = 140000, 32768, 64                       # 4.6e9 elements of bf16
    table = torch.zeros(rows, hidden, dtype=BF16, device=DEV)
    ids = torch.arange(n, device=DEV) + rows - n
    ids[0] = 3
    table[ids] = normal(90, (n, hidden), 1.0, BF16)
    out = torch.empty(n, hidden, dtype=BF16, device=DEV)
    dte.dte_embedding_forward(table, ids, out)
    assert torch.equal(out, table[ids])
    dout = normal(91, (n, hidden), 1.0, BF16)
    table.fill_(1.0)
    dte.dte_embedding_backward(dout, ids, table, workspace(dte.dte_embedding_backward_workspace_bytes(n, hidden)))
    assert torch.equal(table[ids], dout)
    assert int(torch.count_nonzero(table[4:rows - n])) == 0 and int(torch.count_nonzero(table[:3])) == 0


def test_norm_of_more_than_2_to_the_32_elements():
    rows, cols = 1100000, 4096
    x = torch.empty(rows, cols, dtype=BF16, device=DEV)
    tail = normal(92, (300, cols), 1.0, BF16, 0.5)
    x.fill_(0.25)
    x[-300:] = tail
    out, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    dte.dte_norm_forward(x, None, None, out, mean, rstd, 1e-5)
    small, m2, r2 = torch.empty_like(tail), torch.empty(300, device=DEV), torch.empty(300, device=DEV)
    dte.dte_norm_forward(tail, None, None, small, m2, r2, 1e-5)
    assert torch.equal(out[-300:], small) and torch.equal(rstd[-300:], r2) and bool((out[:-300] == 0).all())
    dw, dw2 = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    dx2 = torch.empty_like(tail)
    ws = workspace(dte.dte_norm_backward_workspace_bytes(rows, cols))
    out[:-300] = 0                                            # as dout: nothing but the last rows counts
    dx = torch.empty_like(x)
    dte.dte_norm_backward(out, x, None, mean, rstd, dx, dw, None, ws)
    dte.dte_norm_backward(small, tail, None, m2, r2, dx2, dw2, None, ws)
    assert torch.equal(dx[-300:], dx2) and bool((dx[:-300] == 0).all())
    assert_within(dw, dw2.to(F64), 2 * 340 * E * (small.to(F64).abs() * (tail.to(F64).abs() + 1) * 2).sum(0), "dweight")


def test_head_with_more_than_2_to_the_31_weights():
    tokens, vocab, hidden = 40, 560000, 4096                  # 2.3e9 elements
    w = torch.zeros(vocab, hidden, dtype=BF16, device=DEV)
    x = normal(93, (tokens, hidden), 1.0, BF16)
    hot = torch.arange(tokens, device=DEV) + vocab - tokens
    w[hot] = normal(94, (tokens, hidden), 0.03, BF16)
    lse, tl, loss = run_forward(x, w, hot)
    z = x.to(F64) @ w[hot].to(F64).T
    want = torch.logsumexp(torch.cat([z, torch.full((tokens, 1), math.log(vocab - tokens), dtype=F64, device=DEV)], 1), 1)
    dz = (hidden / 16 + 16) * 2.0 ** -23 * (x.to(F64).abs() @ w[hot].to(F64).abs().T)
    assert_within(lse, want, dz.amax(1) + 2.0 ** -20 + 64 * E * want.abs(), "lse")
    dloss = normal(95, (tokens,))
    dx, dw = run_backward(x, w, hot, lse, dloss)
    p = torch.exp(z - lse.to(F64)[:, None]) * dloss.to(F64)[:, None]
    g = p - torch.diag(dloss.to(F64))
    wdx, wdw = g @ w[hot].to(F64), g.T @ x.to(F64)
    rel = 2.0 ** -8 + 2 * dz + 2.0 ** -18
    mx = (p.abs() * rel) @ w[hot].to(F64).abs() + (tokens + 100) * 2.0 ** -23 * (g.abs() @ w[hot].to(F64).abs())
    mw = (p.abs() * rel).T @ x.to(F64).abs() + (tokens + 100) * 2.0 ** -23 * (g.abs().T @ x.to(F64).abs())
    assert_within(dx, wdx, mx + U[BF16] * wdx.abs() * 1.01, "dx")
    assert_within(dw[hot], wdw, mw + U[BF16] * wdw.abs() * 1.01, "dweight")
    # a row of zeros elsewhere: the sum over tokens of dloss / (sum of exponentials) x
    far = (dloss.to(F64) * torch.exp(-lse.to(F64))) @ x.to(F64)
    size = (dloss.to(F64).abs() * torch.exp(-lse.to(F64))) @ x.to(F64).abs()
    assert_within(dw[12345], far, size * 2.0 ** -7 + U[BF16] * far.abs() * 1.01, "dweight of a row far below 2^31")


# ---- streams, graphs and refusals ------------------------------------------------------------------------------

def test_operators_run_on_a_side_stream_and_inside_a_graph():
    tokens, vocab, hidden = 48, 500, 64
    x, w, t = head_case(tokens, vocab, hidden, 80, 0.2)
    ids = randint(81, 0, vocab, tokens)
    n = torch.empty_like(x)
    e = torch.empty_like(x)
    rstd, lse, loss, dloss = (torch.empty(tokens, device=DEV) for _ in range(4))
    dloss.fill_(1.0 / tokens)
    dn, de, dh, dt = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    dnw = torch.empty(hidden, device=DEV)
    ws = workspace(max(dte.dte_linear_ce_backward_workspace_bytes(tokens, vocab, hidden),
                       dte.dte_linear_ce_forward_workspace_bytes(tokens, vocab, hidden),
                       dte.dte_embedding_backward_workspace_bytes(tokens, hidden), dte.dte_norm_backward_workspace_bytes(tokens, hidden)))

    def step():
        dte.dte_embedding_forward(w, ids, e)
        dte.dte_norm_forward(e, None, None, n, None, rstd, 1e-6, rms=True)
        dte.dte_linear_ce_forward(n, w, t, lse, None, loss, ws)
        dte.dte_linear_ce_backward(n, w, t, lse, dloss, dn, dh, ws)
        dte.dte_norm_backward(dn, e, None, None, rstd, de, dnw, None, ws, rms=True)
        dte.dte_embedding_backward(de, ids, dt, ws)
        return [v.clone() for v in (loss, dh, dnw, dt)]

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for v in (loss, dh, dnw, dt):
            v.fill_(7)
        got = step()
        side.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
    ids.copy_(randint(82, 0, vocab, tokens))
    for _ in range(2):
        for v in (loss, dh, dnw, dt):
            v.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        replayed = [v.clone() for v in (loss, dh, dnw, dt)]
        for a, b in zip(replayed, step()):
            assert torch.equal(a, b)


def refused(match, call):
    with pytest.raises(dte.DteError, match=match) as e:
        call()
    return e.value.status


def test_refusals():
    t4, ids = torch.zeros(4, 8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    out = torch.zeros(4, 8, device=DEV)
    ws = workspace(1 << 20)
    f, v4 = dte.dte_embedding_forward, torch.zeros(4, device=DEV)
    assert refused("float32 or bfloat16", lambda: f(t4.double(), ids, out)) == 1
    assert refused("int32 or int64", lambda: f(t4, ids.float(), out)) == 1
    assert refused("ids.count x table.cols", lambda: f(t4, ids[:3], out)) == 1
    assert refused("ids.count x table.cols", lambda: f(t4, ids, torch.zeros(4, 9, device=DEV))) == 1
    assert refused("last dimension", lambda: f(t4.t(), ids, out)) == 1
    assert refused("rows overlap", lambda: f(t4, ids, out[:1].expand(4, 8))) == 1
    assert refused("inside the vocabulary", lambda: f(t4, ids, out, row_start=3, vocab=6)) == 1
    assert refused("negative", lambda: f(t4, ids, out, row_start=-1)) == 1
    assert refused("finite", lambda: f(t4, ids, out, scale=float("nan"))) == 1
    assert refused("CUDA device", lambda: f(t4.cpu(), ids, out)) == 1
    assert refused("CUDA device", lambda: f(t4, ids.cpu(), out)) == 1
    assert refused("too small", lambda: dte.dte_embedding_backward(out, ids, t4, ws[:64])) == 3
    assert refused("256-byte aligned", lambda: dte.dte_embedding_backward(out, ids, t4, ws[8:])) == 1
    n = dte.dte_norm_forward
    assert refused("shape and type", lambda: n(t4, None, None, out.bfloat16(), None, None, 1e-6)) == 1
    assert refused("eps", lambda: n(t4, None, None, out, None, None, -1.0)) == 1
    assert refused("8 values", lambda: n(t4, torch.ones(7, device=DEV), None, out, None, None, 1e-6)) == 1
    assert refused("one type", lambda: n(t4, torch.ones(8, device=DEV), torch.ones(8, device=DEV, dtype=BF16), out, None, None, 1e-6)) == 1
    assert refused("4 values", lambda: n(t4, None, None, out, None, torch.ones(3, device=DEV), 1e-6)) == 1
    assert refused("mean / rstd", lambda: dte.dte_norm_backward(out, t4, None, None, v4, out, None, None, ws)) == 1
    assert refused("too small", lambda: dte.dte_norm_backward(out, t4, None, v4, v4, out, torch.zeros(8, device=DEV), None, None)) == 3
    x, w = torch.zeros(4, 16, dtype=BF16, device=DEV), torch.zeros(10, 16, dtype=BF16, device=DEV)
    lse = torch.zeros(4, device=DEV)
    c = dte.dte_linear_ce_forward
    assert refused("BF16", lambda: c(x.float(), w, ids, lse, None, None, ws)) == 1
    assert refused("multiple of 8", lambda: c(x[:, :12], w[:, :12], ids, lse, None, None, ws)) == 1
    assert refused("16-byte aligned", lambda: c(x[:, :8], w[:, 4:12], ids, lse, None, None, ws)) == 1
    assert refused("logit_scale", lambda: c(x, w, ids, lse, None, None, ws, logit_scale=0.0)) == 1
    assert refused("targets.count", lambda: c(x[:3], w, ids, lse, None, None, ws)) == 1
    assert refused("no rows", lambda: c(x, w[:0], ids, lse, None, None, ws)) == 1
    assert refused("too small", lambda: c(x, w, ids, lse, None, None, ws[:1024])) == 3
    b = dte.dte_linear_ce_backward
    assert refused("x's shape", lambda: b(x, w, ids, lse, lse, x.float(), None, ws)) == 1
    assert refused("weight's shape", lambda: b(x, w, ids, lse, lse, None, w[:9], ws)) == 1
    small = dte.dte_linear_ce_backward_workspace_min_bytes(4, 10, 16)
    assert refused("too small", lambda: b(x, w, ids, lse, lse, None, torch.zeros_like(w), ws[:small - 256])) == 3
    torch.cuda.synchronize()


def test_a_device_that_does_not_exist_is_refused_and_leaves_nothing_behind():
    L, none = dte.lib(), 63
    assert torch.cuda.device_count() <= none
    stream = torch.cuda.current_stream().cuda_stream
    n, v, h = 4, 10, 16
    t, x, w = randint(160, 0, v, n), normal(161, (n, h), 1.0, BF16), normal(162, (v, h), 1.0, BF16)
    out, dw, s = torch.full_like(x, 7.0), torch.full_like(w, 7.0), torch.full((n,), 7.0, device=DEV)
    ws = workspace(1 << 26)
    mat = lambda a: ops._pack_matrix(a.data_ptr(), *a.shape, a.shape[1], ops.DTE_BF16, 0)                       # noqa: E731
    i, size = ops._pack_ids(t.data_ptr(), n, ops.DTE_I64, 0), ws.numel()
    m, o, g, p, q = mat(x), mat(out), mat(dw), s.data_ptr(), ws.data_ptr()
    calls = (lambda d: L.dte_embedding_forward(mat(w), i, 0, v, 1.0, o, None, d, stream),
             lambda d: L.dte_embedding_backward(m, i, 0, v, 1.0, 0, g, q, size, None, d, stream),
             lambda d: L.dte_norm_forward(m, None, None, 0, 1, 1e-6, o, None, p, d, stream),
             lambda d: L.dte_norm_backward(m, m, None, 0, 1, None, p, 0, o, None, None, None, 0, d, stream),
             lambda d: L.dte_linear_ce_forward(m, mat(w), i, 0, v, 1.0, p, None, None, q, size, None, d, stream),
             lambda d: L.dte_linear_ce_backward(m, mat(w), i, 0, v, 1.0, p, p, 0, o, g, q, size, None, d, stream))
    for k, call in enumerate(calls):
        for a in (out, dw, s):
            a.fill_(7.0)
        torch.cuda.synchronize()
        assert call(none) == 1 and b"device" in L.dte_last_error(), k
        torch.cuda.synchronize()
        assert all(bool((a == 7.0).all()) for a in (out, dw, s)), k
        assert call(0) == 0, (k, L.dte_last_error())
        torch.cuda.synchronize()
