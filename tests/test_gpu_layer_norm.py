"""Layer norm, forward and backward, against its definition in 64 bits.

Tolerances come from the arithmetic, before any run.  u = 2^-24 is fp32's unit
roundoff.  A sum whose longest chain of additions is D is within D u of the sum
of the terms' magnitudes; D is at most 48 (32 elements of a lane and the
joining of lanes and waves) plus cols / 1024 (the elements of a lane in the
long rows' form).  A sum over R rows in any order is within R u.  Results in
bf16 are rounded once more, by at most 2^-9 of their size.
"""
import numpy as np
import pytest

from helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}       # rounding to the output type (twice the unit, for the sum's own)
TINY = 1e-37                                        # below the normal numbers


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_04676_amd as S
    return S


def depth(cols):
    return 48 + cols // 1024


def matrix(rows, cols, dtype, seed, scale=1.0, shift=0.0, pad=0, offset=0):
    """Rows inside a wider buffer that starts `offset` elements late; the
    buffer's other elements are NaN, so that a read outside the rows shows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((offset + rows * (cols + pad) + 16,), float("nan"), dtype=DT[dtype], device="cuda")
    m = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn((rows, cols), generator=g, device="cuda") * scale + shift)
    return m


def vector(n, dtype, seed, scale, shift):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, generator=g, device="cuda") * scale + shift).to(DT[dtype])


def untouched(m):
    """The elements of m's buffer outside m are still NaN."""
    buf = torch.empty(0, dtype=m.dtype, device=m.device).set_(m.untyped_storage())
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask.as_strided(m.shape, m.stride(), m.storage_offset()).fill_(False)
    return bool(buf[mask].isnan().all())


def within(got, exp, bound, what):
    err = (got.double() - exp).abs()
    bad = ~(err <= bound)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound).nan_to_num(1e9).max()):.3g} times the bound"


def forward_bounds(x, w, b, eps, out):
    """The definition in 64 bits and what fp32 arithmetic may be off it."""
    C = x.shape[1]
    x = x.double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = d.square().mean(1, keepdim=True)
    rstd = 1.0 / (var + eps).sqrt()
    h = d * rstd
    w = torch.ones(C, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(C, dtype=torch.float64, device=x.device) if b is None else b.double()
    y = h * w + b
    D = depth(C) + 4
    em = D * U * x.abs().mean(1, keepdim=True) + U * mean.abs()
    # the deviations: each off by em and a rounding, their squares' sum by D u more
    ev = 2 * em * d.abs().mean(1, keepdim=True) + em * em + (D + 4) * U * var
    # var + eps may be off by ev and two roundings; 1 / sqrt halves that (for any size of it)
    rel = (ev + 2 * U * (var + eps)) / (var + eps)
    er = torch.where(rel < 0.5, rel, torch.full_like(rel, 1e30)) * rstd + 3 * U * rstd
    ey = w.abs() * (rstd * (em + U * d.abs()) + d.abs() * er + 3 * U * h.abs()) + 2 * U * (h * w).abs() + U * b.abs()
    return (mean, em + TINY), (rstd, er), (y, ey + OUT[out] * y.abs() + TINY)


SIZES = [(1, 1), (5, 1), (1, 64), (3, 7), (3, 65), (2, 63), (257, 64), (130, 128), (67, 200), (33, 512), (19, 513),
         (9, 1600), (5, 2048), (3, 2049), (6, 4096), (4, 4099), (3, 8192), (2, 8193), (3, 16384), (2, 16385), (2, 32768),
         (2, 32769), (1, 70_001), (5000, 96), (2500, 1600), (70_000, 3)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_forward(S, rows, cols, dtype, wdtype):
    log(f"layer norm {rows}x{cols} {dtype} {wdtype}")
    seed = rows * 7 + cols
    pad, offset = (0, 0) if cols % 2 == 0 else (seed % 5, seed % 3)
    x = matrix(rows, cols, dtype, seed, 2.0, 0.7, pad, offset)
    y = matrix(rows, cols, dtype, seed + 1, 1.0, 0.0, pad + 1, 1)
    w, b = vector(cols, wdtype, seed + 2, 0.3, 1.0), vector(cols, wdtype, seed + 3, 0.3, 0.1)
    mean, rstd = torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
    S.spccl_layer_norm(x, w, b, y, mean, rstd, 1e-5)
    torch.cuda.synchronize()
    (m, em), (r, er), (e, ee) = forward_bounds(x, w, b, 1e-5, dtype)
    within(mean[:, None], m, em, "mean")
    within(rstd[:, None], r, er, "rstd")
    within(y, e, ee, "y")
    assert untouched(x) and untouched(y)


@pytest.mark.parametrize("cols", [100, 1600, 5000, 40_000])
def test_forward_without_weight_bias_or_statistics(S, cols):
    log(f"layer norm without weights, {cols}")
    x, y = matrix(4, cols, "bf16", cols, 1.0), matrix(4, cols, "bf16", 1)
    for w, b in ((None, None), (vector(cols, "f32", 3, 1.0, 0.0), None), (None, vector(cols, "bf16", 4, 1.0, 0.0))):
        S.spccl_layer_norm(x, w, b, y)
        torch.cuda.synchronize()
        e, ee = forward_bounds(x, w, b, 1e-5, "bf16")[2]
        within(y, e, ee, "y")


@pytest.mark.parametrize("cols", [64, 1000, 3000, 9000, 33_000])
def test_forward_in_place_and_far_from_zero(S, cols):
    """y may be x; a mean 1000 times the spread costs the mean's rounding, not
    the spread's precision."""
    log(f"layer norm in place, {cols}")
    x = matrix(3, cols, "f32", cols, 1.0, 1000.0)
    e, ee = forward_bounds(x, None, None, 1e-5, "f32")[2]
    S.spccl_layer_norm(x, None, None, x)
    torch.cuda.synchronize()
    within(x, e, ee, "y")


def test_rows_that_are_constant_infinite_or_nan(S):
    """A constant row has no deviation: h = 0 and y = bias.  A row that holds an
    infinity or a NaN is NaN, and no other row is."""
    log("layer norm special rows")
    for cols in (96, 1600, 5000, 40_000):
        x = matrix(5, cols, "f32", 5, 1.0)
        x[1] = 0.0
        x[2] = 3.0
        x[3, cols // 2] = float("inf")
        x[4, 0] = float("nan")
        b = vector(cols, "f32", 2, 1.0, 0.0)
        y, mean, rstd = torch.empty_like(x), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
        S.spccl_layer_norm(x, None, b, y, mean, rstd)
        torch.cuda.synchronize()
        assert torch.equal(y[1], b) and torch.equal(y[2], b)
        assert bool(y[3].isnan().all()) and bool(y[4].isnan().all())
        assert bool(y[:3].isfinite().all()) and bool(rstd[:3].isfinite().all())


def backward_bounds(dy, x, w, mean, rstd, dtype):
    rows, C = x.shape
    dy, x = dy.double(), x.double()
    mean, rstd = mean.double()[:, None], rstd.double()[:, None]
    w = torch.ones(C, dtype=torch.float64, device=x.device) if w is None else w.double()
    h = (x - mean) * rstd
    g = dy * w
    s1, s2 = (g * h).mean(1, keepdim=True), g.mean(1, keepdim=True)
    dx = rstd * (g - s2 - h * s1)
    D = depth(C) + 8
    e1, e2 = D * U * (g * h).abs().mean(1, keepdim=True), D * U * g.abs().mean(1, keepdim=True)
    ex = rstd.abs() * (e2 + h.abs() * e1 + 8 * U * (g.abs() + s2.abs() + (h * s1).abs()))
    dw, db = (dy * h).sum(0), dy.sum(0)
    ew, eb = (rows + 8) * U * (dy * h).abs().sum(0), (rows + 8) * U * dy.abs().sum(0)
    return (dx, ex + OUT[dtype] * dx.abs() + TINY), (dw, ew + TINY), (db, eb + TINY)


def scratch_for(S, rows, cols):
    need = S.spccl_layer_norm_scratch_bytes(rows, cols)
    t = torch.full((max(16, need) + 64,), 0xFF, dtype=torch.uint8, device="cuda")     # NaN where not written
    return t[:max(16, need)], t


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype,wdtype,gdtype,accumulate", [("f32", "f32", "f32", False), ("f32", "bf16", "bf16", True),
                                                            ("bf16", "bf16", "f32", True), ("bf16", "f32", "bf16", False)])
def test_backward(S, rows, cols, dtype, wdtype, gdtype, accumulate):
    log(f"layer norm backward {rows}x{cols} {dtype} {wdtype} {gdtype} {accumulate}")
    seed = rows * 7 + cols
    pad, offset = (0, 0) if cols % 2 == 0 else (seed % 5, seed % 3)
    x = matrix(rows, cols, dtype, seed, 2.0, 0.7, pad, offset)
    dy = matrix(rows, cols, dtype, seed + 1, 1.0, 0.1, pad + 2, 1)
    dx = matrix(rows, cols, dtype, seed + 2, 1.0, 0.0, 1, 2)
    w = vector(cols, wdtype, seed + 3, 0.3, 1.0)
    mean = x.float().mean(1)
    rstd = 1.0 / (x.float().var(1, unbiased=False) + 1e-5).sqrt()
    dw, db = vector(cols, gdtype, seed + 4, 1.0, 0.0), vector(cols, gdtype, seed + 5, 1.0, 0.0)
    before = dw.double(), db.double()
    scratch, whole = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, scratch, accumulate)
    torch.cuda.synchronize()
    (ex, bx), (ew, bw), (eb, bb) = backward_bounds(dy, x, w, mean, rstd, dtype)
    if accumulate:
        ew, eb = ew + before[0], eb + before[1]
        bw, bb = bw + 2 * U * ew.abs(), bb + 2 * U * eb.abs()
    within(dx, ex, bx, "dx")
    within(dw, ew, bw + OUT[gdtype] * ew.abs(), "dweight")
    within(db, eb, bb + OUT[gdtype] * eb.abs(), "dbias")
    assert untouched(x) and untouched(dy) and untouched(dx)
    assert bool((whole[scratch.numel():] == 0xFF).all())


@pytest.mark.parametrize("rows,cols", [(128, 300), (129, 300), (192, 257), (193, 4100), (512, 100), (513, 100), (1024, 1030),
                                       (1025, 1030), (130, 20_001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_around_the_strips_of_rows(S, rows, cols, dtype):
    """Row counts where a few rows' launch takes another strip or ends, also in place."""
    log(f"layer norm backward strips {rows}x{cols} {dtype}")
    x, dy = matrix(rows, cols, dtype, 1, 2.0, 0.5), matrix(rows, cols, dtype, 2)
    w = vector(cols, "f32", 3, 0.3, 1.0)
    mean = x.float().mean(1)
    rstd = 1.0 / (x.float().var(1, unbiased=False) + 1e-5).sqrt()
    (ex, bx), (ew, bw), (eb, bb) = backward_bounds(dy, x, w, mean, rstd, dtype)
    first = None
    for over in ("apart", "x", "dy"):
        a, b = dy.clone(), x.clone()
        dx = {"apart": torch.empty_like(x), "x": b, "dy": a}[over]
        dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        scratch, whole = scratch_for(S, rows, cols)
        S.spccl_layer_norm_backward(a, b, w, mean, rstd, dx, dw, db, scratch)
        torch.cuda.synchronize()
        within(dx, ex, bx, "dx")
        within(dw, ew, bw + OUT["f32"] * ew.abs(), "dweight")
        within(db, eb, bb + OUT["f32"] * eb.abs(), "dbias")
        assert bool((whole[scratch.numel():] == 0xFF).all())
        first = first or (dx.clone(), dw, db)
        assert all(torch.equal(p, q) for p, q in zip(first, (dx, dw, db)))


@pytest.mark.parametrize("rows,cols", [(70, 1600), (40, 128), (12, 5000), (9, 20_000)])
def test_backward_of_parts_in_place_and_twice(S, rows, cols):
    """Each gradient alone, dx over dy or over x, and equal bits from equal calls."""
    log(f"layer norm backward parts {rows}x{cols}")
    x, dy = matrix(rows, cols, "f32", 1, 2.0, 0.5), matrix(rows, cols, "f32", 2)
    w = vector(cols, "f32", 3, 0.3, 1.0)
    mean = x.mean(1)
    rstd = 1.0 / (x.var(1, unbiased=False) + 1e-5).sqrt()
    new = lambda: (torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda"))  # noqa: E731
    dx, dw, db = new()
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, scratch)
    for which in range(5):
        dx2, dw2, db2 = new()
        if which == 0:
            S.spccl_layer_norm_backward(dy, x, w, mean, rstd, dx2, None, None)
            assert torch.equal(dx, dx2)
        elif which == 1:
            S.spccl_layer_norm_backward(dy, x, w, mean, rstd, None, dw2, db2, scratch)
            assert torch.equal(dw, dw2) and torch.equal(db, db2)
        elif which == 2:
            S.spccl_layer_norm_backward(dy, x, w, mean, rstd, dx2, dw2, None, scratch)
            assert torch.equal(dw, dw2) and torch.equal(dx, dx2)
        else:
            a, b = dy.clone(), x.clone()
            over = a if which == 3 else b
            S.spccl_layer_norm_backward(a, b, w, mean, rstd, over, dw2, db2, scratch)
            assert torch.equal(over, dx) and torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("rows,cols", [(133, 64), (133, 63), (261, 1000), (515, 2048), (259, 4096), (300, 12_000), (131, 20_000)])
@pytest.mark.parametrize("over", ["x", "dy", "apart"])
def test_a_nan_gradient_stays_in_its_row_and_column(S, rows, cols, over):
    """A NaN in dy's last row: that row of dx and that column's sums are NaN and
    nothing else, wherever dx is written and however the rows fill the blocks."""
    log(f"layer norm backward nan {rows}x{cols} {over}")
    x, dy = matrix(rows, cols, "f32", 1, 2.0, 0.5), matrix(rows, cols, "f32", 2)
    mean = x.mean(1)
    rstd = 1.0 / (x.var(1, unbiased=False) + 1e-5).sqrt()
    dy[rows - 1, 5] = float("nan")
    dx = {"x": x, "dy": dy, "apart": torch.empty_like(x)}[over]
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, None, mean, rstd, dx, dw, db, scratch)
    torch.cuda.synchronize()
    assert bool(dx[:rows - 1].isfinite().all()) and bool(dx[rows - 1].isnan().all())
    for g in (dw, db):
        assert g.isnan().nonzero().flatten().tolist() == [5]


def test_no_rows(S):
    log("layer norm without rows")
    x = torch.empty((0, 80), device="cuda")
    one = torch.empty(0, device="cuda")
    S.spccl_layer_norm(x, None, None, torch.empty_like(x), one, one)
    for gdtype in DT:
        dw, db = vector(80, gdtype, 1, 1.0, 0.0), vector(80, gdtype, 2, 1.0, 0.0)
        keep = dw.clone()
        S.spccl_layer_norm_backward(x, x, None, one, one, torch.empty_like(x), dw, db, None, accumulate=True)
        torch.cuda.synchronize()
        assert torch.equal(dw, keep)
        S.spccl_layer_norm_backward(x, x, None, one, one, torch.empty_like(x), dw, db, None)
        torch.cuda.synchronize()
        assert not bool(dw.any()) and not bool(db.any())


def test_rows_past_32_bit_offsets(S):
    """Rows 2^31 elements apart: their offsets pass 32 bits in elements and bytes."""
    log("layer norm far rows")
    rows, cols, pitch = 3, 300, 1 << 31
    buf = torch.empty(2 * pitch + cols, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, cols), (pitch, 1))
    x.copy_(matrix(rows, cols, "bf16", 3, 2.0, 0.5))
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    S.spccl_layer_norm(x, None, None, y, mean, rstd)
    torch.cuda.synchronize()
    (_, _), (_, _), (e, ee) = forward_bounds(x, None, None, 1e-5, "bf16")
    within(y, e, ee, "y")
    dy = matrix(rows, cols, "bf16", 4)
    (ex, bx), (ew, bw), (eb, bb) = backward_bounds(dy, x, None, mean, rstd, "bf16")
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, None, mean, rstd, x, dw, db, scratch)
    torch.cuda.synchronize()
    within(x, ex, bx, "dx")
    within(dw, ew, bw + OUT["f32"] * ew.abs(), "dweight")


@pytest.mark.parametrize("dtype,cols", [("bf16", 3), ("f32", 2)])
def test_more_rows_than_one_grid_of_long_rows(S, dtype, cols):
    """Rows shorter than a vector take a block each: more of them than a grid of
    such blocks may hold."""
    log(f"layer norm many short rows {dtype} {cols}")
    rows = (1 << 22) + 77
    x, dy = matrix(rows, cols, dtype, 1, 2.0, 0.5), matrix(rows, cols, dtype, 2)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    S.spccl_layer_norm(x, None, None, y, mean, rstd)
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, None, mean, rstd, dx, dw, db, scratch)
    torch.cuda.synchronize()
    (m, em), (r, er), (e, ee) = forward_bounds(x, None, None, 1e-5, dtype)
    within(mean[:, None], m, em, "mean")
    within(rstd[:, None], r, er, "rstd")
    within(y, e, ee, "y")
    (ex, bx), (ew, bw), (eb, bb) = backward_bounds(dy, x, None, mean, rstd, dtype)
    within(dx, ex, bx, "dx")
    within(dw, ew, bw + OUT["f32"] * ew.abs(), "dweight")
    within(db, eb, bb + OUT["f32"] * eb.abs(), "dbias")


def test_gradient_against_differences(S):
    """Central differences of the forward kernel along random directions.  The
    step's own error is that of the same differences in 64 bits; the kernel's
    adds its forward bound twice over the step."""
    log("layer norm differences")
    rows, cols, step = 6, 700, 2.0 ** -6
    x, dy = matrix(rows, cols, "f32", 11, 1.0, 0.2), matrix(rows, cols, "f32", 12)
    w, b = vector(cols, "f32", 13, 0.3, 1.0), vector(cols, "f32", 14, 0.3, 0.0)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y = torch.empty((rows, cols), device="cuda")

    def kernel(x_, w_, b_):
        S.spccl_layer_norm(x_, w_, b_, y, mean, rstd)
        return (y.double() * dy.double()).sum()

    def exact(x_, w_, b_):
        (_, _), (_, _), (e, ee) = forward_bounds(x_, w_, b_, 1e-5, "f32")
        return (e * dy.double()).sum(), (ee * dy.double().abs()).sum()

    kernel(x, w, b)
    mean0, rstd0 = mean.clone(), rstd.clone()
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, w, mean0, rstd0, dx, dw, db, scratch)
    (ex, bx), (ew, bw), (eb, bb) = backward_bounds(dy, x, w, mean0, rstd0, "f32")
    # the statistics themselves are fp32: the analytic gradient's own share
    share = 64 * U
    for grad, bound, at in ((dx, bx, 0), (dw, bw, 1), (db, bb, 2)):
        args = [x.contiguous(), w, b]
        g = torch.Generator(device="cuda").manual_seed(20 + at)
        v = torch.randn(args[at].shape, generator=g, device="cuda")
        plus, minus = list(args), list(args)
        plus[at], minus[at] = args[at] + step * v, args[at] - step * v
        v64 = (plus[at].double() - minus[at].double()) / (2 * step)      # the step as it was rounded
        diff = (kernel(*plus) - kernel(*minus)) / (2 * step)
        p, m = exact(*plus), exact(*minus)
        exact64 = [t.double().requires_grad_(i == at) for i, t in enumerate(args)]
        x_, w_, b_ = exact64
        d = x_ - x_.mean(1, keepdim=True)
        f = ((d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * w_ + b_) * dy.double()).sum()
        true = (torch.autograd.grad(f, exact64[at])[0] * v64).sum()
        curve = abs(float((p[0] - m[0]) / (2 * step) - true))
        tol = curve + float((p[1] + m[1]) / (2 * step)) + float((bound * v64.abs()).sum()) \
            + share * float((grad.double() * v64).abs().sum())
        assert abs(float((grad.double() * v64).sum() - diff)) <= tol


def test_on_another_stream_and_in_a_graph(S):
    """Replays of a captured forward and backward pass, with other work between
    them, equal the eager results of the same inputs."""
    log("layer norm graph")
    rows, cols = 300, 1600
    x, dy = matrix(rows, cols, "bf16", 1, 2.0), matrix(rows, cols, "bf16", 2)
    w, b = vector(cols, "f32", 3, 0.3, 1.0), vector(cols, "f32", 4, 0.3, 0.0)
    new = lambda: [torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"),  # noqa: E731
                   torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")]
    scratch, _ = scratch_for(S, rows, cols)

    def both(o, stream=None):
        S.spccl_layer_norm(x, w, b, o[0], o[1], o[2], 1e-5, stream=stream)
        S.spccl_layer_norm_backward(dy, x, w, o[1], o[2], o[3], o[4], o[5], scratch, stream=stream)

    out = new()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(out, side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out)
    for k in range(4):
        x.mul_(1.01)
        dy.add_(0.01)
        for t in out:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = new()
        both(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, eager)), k


def test_binding_refuses(S):
    x = torch.zeros((4, 8), device="cuda")
    one = torch.zeros(4, device="cuda")
    w = torch.zeros(8, device="cuda")
    bad = [lambda: S.spccl_layer_norm(x.t(), w, w, x), lambda: S.spccl_layer_norm(x, w[:7], w, x),
           lambda: S.spccl_layer_norm(x, w, w.bfloat16(), x), lambda: S.spccl_layer_norm(x, w, w, x.bfloat16()),
           lambda: S.spccl_layer_norm(x, w, w, x, one.double(), one), lambda: S.spccl_layer_norm(x[0], w, w, x[0]),
           lambda: S.spccl_layer_norm_backward(x, x[:2], w, one, one, None, None, None),
           lambda: S.spccl_layer_norm_backward(x, x, w, one[:2], one, x, None, None)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        S.spccl_layer_norm(x.half(), None, None, x.half())
    with pytest.raises(S.SpcclError):
        S.spccl_layer_norm_backward(x, x, w, one, one, None, w.clone(), w.clone(), None)     # no scratch


@pytest.mark.parametrize("rows,cols,dtype", [(1, 65, "f32"), (3, 126, "f32"), (3, 126, "bf16"), (130, 1001, "bf16"),
                                             (515, 64, "f32"), (515, 127, "f32"), (1031, 126, "bf16"), (1031, 1000, "bf16"),
                                             (517, 1028, "f32"), (515, 16_386, "f32"), (1025, 16_388, "bf16"),
                                             (1025, 3, "bf16")])
@pytest.mark.parametrize("over", ["apart", "x", "dy"])
def test_elements_that_do_not_exist_add_nothing(S, rows, cols, dtype, over):
    """Constant rows far from zero: mean and rstd are finite, their product is
    not, and no element deviates, so dweight is 0 and the rest finite.  Places
    past a row's end and groups of lanes past the last row hold zeros, which do
    deviate from that mean; they must not count."""
    log(f"layer norm backward constant rows {rows}x{cols} {dtype} {over}")
    x, dy = matrix(rows, cols, dtype, 1), matrix(rows, cols, dtype, 2)
    x.fill_(2.0 ** 120)
    w = vector(cols, "f32", 3, 0.3, 1.0)
    mean = torch.full((rows,), 2.0 ** 120, device="cuda")
    rstd = torch.full((rows,), 1e-5 ** -0.5, device="cuda")
    assert not bool((mean * rstd).isfinite().any())
    (ex, bx), (ew, bw), (eb, bb) = backward_bounds(dy, x, w, mean, rstd, dtype)
    dx = {"apart": torch.empty_like(x), "x": x, "dy": dy}[over]
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, scratch)
    torch.cuda.synchronize()
    within(dx, ex, bx, "dx")
    assert not bool(dw.any())
    within(db, eb, bb + OUT["f32"] * eb.abs(), "dbias")


def short_rows_bounds(rows, dy, h):
    """The columns' sums in 64 bits, and their bounds.  2^17 rows are worked on
    at a time, so a lane adds rows / 2^17 terms one after another; lanes, waves
    and blocks are joined in at most 56 steps, and h has 3 roundings."""
    depth = 64 + rows // (1 << 17)
    ew, eb = (dy * h).sum(0), dy.sum(0)
    return (ew, depth * U * (dy * h).abs().sum(0) + TINY), (eb, depth * U * dy.abs().sum(0) + TINY)


@pytest.mark.parametrize("rows", [513, 1025, 4099, 70_001, (1 << 17) + 1, (1 << 22) + 77])
@pytest.mark.parametrize("dtype,cols", [("f32", 1), ("f32", 2), ("f32", 3), ("bf16", 1), ("bf16", 2), ("bf16", 5), ("bf16", 7)])
@pytest.mark.parametrize("gdtype,accumulate", [("f32", False), ("f32", True), ("bf16", True)])
def test_sums_over_short_rows(S, rows, dtype, cols, gdtype, accumulate):
    """Gradients of the same sign in every row, where a long chain of additions
    would round the same way again and again."""
    log(f"layer norm backward short rows {rows}x{cols} {dtype} {gdtype} {accumulate}")
    x, dy = matrix(rows, cols, dtype, 1, 0.3, 0.0, 1, 1), matrix(rows, cols, dtype, 2, 0.0, 0.1, 2)
    mean, rstd = torch.full((rows,), -1.7, device="cuda"), torch.full((rows,), 0.7, device="cuda")
    x[rows // 2:] = 0.3
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    (ew, bw), (eb, bb) = short_rows_bounds(rows, dy.double(), h)
    dw, db = vector(cols, gdtype, 4, 10.0, 0.0), vector(cols, gdtype, 5, 10.0, 0.0)
    if accumulate:
        ew, eb = ew + dw.double(), eb + db.double()
        bw, bb = bw + 2 * U * ew.abs(), bb + 2 * U * eb.abs()
    scratch, whole = scratch_for(S, rows, cols)
    again = dw.clone(), db.clone()
    S.spccl_layer_norm_backward(dy, x, None, mean, rstd, None, dw, db, scratch, accumulate)
    S.spccl_layer_norm_backward(dy, x, None, mean, rstd, None, *again, scratch, accumulate)
    torch.cuda.synchronize()
    within(dw, ew, bw + OUT[gdtype] * ew.abs(), "dweight")
    within(db, eb, bb + OUT[gdtype] * eb.abs(), "dbias")
    assert torch.equal(dw, again[0]) and torch.equal(db, again[1])
    assert bool((whole[scratch.numel():] == 0xFF).all())


def test_sums_over_the_most_rows(S):
    """2^31 - 1 rows of one element: sums past 2^24, where fp32 no longer counts
    in ones.  x and dy share their memory, and so do mean and rstd."""
    log("layer norm backward of 2^31 - 1 rows")
    rows = (1 << 31) - 1
    x = torch.full((rows, 1), 1.5, dtype=torch.bfloat16, device="cuda")
    one = torch.ones(rows, device="cuda")
    dw, db = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    scratch, _ = scratch_for(S, rows, 1)
    S.spccl_layer_norm_backward(x, x, None, one, one, None, dw, db, scratch)
    torch.cuda.synchronize()
    depth = 64 + rows // (1 << 17)
    for got, each in ((dw, 0.75), (db, 1.5)):
        assert abs(float(got) - each * rows) <= depth * U * each * rows


# Widths in every layout of the backward kernel that keeps its rows in registers
# (whole vectors, an odd length, and the widest), and one past the last; rows past
# the few that another kernel takes, and no multiple of what a block holds.
BACK_WIDTHS = [8, 63, 64, 71, 128, 200, 251, 256, 333, 512, 777, 1024, 1111, 1536, 1544, 1999, 2048, 2056, 2500, 3001, 4095, 4096,
               4104, 5001, 6144, 6145, 7000, 8192, 8200, 9999, 12_288, 12_289, 14_336, 16_383, 16_384, 16_385, 16_392]


@pytest.mark.parametrize("cols", BACK_WIDTHS)
@pytest.mark.parametrize("dtype,rows,wdtype,gdtype,accumulate",
                         [("f32", 519, "f32", "f32", False), ("f32", 1031, "bf16", "f32", True),
                          ("bf16", 1031, "f32", "f32", False), ("bf16", 2063, "bf16", "bf16", True)])
@pytest.mark.parametrize("place", ["aligned", "odd pitch", "late"])
def test_backward_in_every_layout(S, cols, dtype, rows, wdtype, gdtype, accumulate, place):
    """Values apart and over x and over dy, from rows that start on 16 bytes and
    from rows that do not."""
    log(f"layer norm backward layouts {rows}x{cols} {dtype} {wdtype} {gdtype} {accumulate} {place}")
    vec = 4 if dtype == "f32" else 8
    # "aligned": every row starts on 16 bytes, whatever its length
    pad, offset = {"aligned": (-cols % vec, 0), "odd pitch": (1 - cols % 2 + 2, 0), "late": (-cols % vec, 1)}[place]
    x, dy = matrix(rows, cols, dtype, cols, 2.0, 0.7, pad, offset), matrix(rows, cols, dtype, cols + 1, 1.0, 0.1, pad, offset)
    w = vector(cols, wdtype, 3, 0.3, 1.0)
    mean = x.float().mean(1)
    rstd = 1.0 / (x.float().var(1, unbiased=False) + 1e-5).sqrt()
    dw0, db0 = vector(cols, gdtype, 4, 1.0, 0.0), vector(cols, gdtype, 5, 1.0, 0.0)
    (ex, bx), (ew, bw), (eb, bb) = backward_bounds(dy, x, w, mean, rstd, dtype)
    if accumulate:
        ew, eb = ew + dw0.double(), eb + db0.double()
        bw, bb = bw + 2 * U * ew.abs(), bb + 2 * U * eb.abs()
    scratch, whole = scratch_for(S, rows, cols)
    first = None
    for over in ("apart", "x", "dy"):
        a, b = (matrix(rows, cols, dtype, 1, 0.0, 0.0, pad, offset).copy_(t) for t in (dy, x))
        dx = {"apart": matrix(rows, cols, dtype, 6, 1.0, 0.0, pad, offset), "x": b, "dy": a}[over]
        dw, db = dw0.clone(), db0.clone()
        S.spccl_layer_norm_backward(a, b, w, mean, rstd, dx, dw, db, scratch, accumulate)
        torch.cuda.synchronize()
        if first is None:
            within(dx, ex, bx, "dx")
            within(dw, ew, bw + OUT[gdtype] * ew.abs(), "dweight")
            within(db, eb, bb + OUT[gdtype] * eb.abs(), "dbias")
            first = dx.clone(), dw, db
        assert all(torch.equal(p, q) for p, q in zip(first, (dx, dw, db)))
        assert untouched(a) and untouched(b) and untouched(dx)
    assert bool((whole[scratch.numel():] == 0xFF).all())


@pytest.mark.parametrize("cols", [64, 63, 1000, 1600, 2048, 3001, 4096, 6000, 8192, 8195, 12_000, 16_384, 16_390])
@pytest.mark.parametrize("dtype,rows", [("f32", 519), ("f32", 4099), ("bf16", 1031), ("bf16", 4099)])
@pytest.mark.parametrize("over", ["x", "dy", "apart"])
def test_a_nan_gradient_stays_in_its_row_and_column_of_many(S, dtype, rows, cols, over):
    """The first and the last row, past the few rows that another kernel takes."""
    log(f"layer norm backward nan {rows}x{cols} {dtype} {over}")
    x, dy = matrix(rows, cols, dtype, 1, 2.0, 0.5), matrix(rows, cols, dtype, 2)
    mean = x.float().mean(1)
    rstd = 1.0 / (x.float().var(1, unbiased=False) + 1e-5).sqrt()
    dy[rows - 1, 5] = float("nan")
    dy[0, cols - 1] = float("nan")
    dx = {"x": x, "dy": dy, "apart": torch.empty_like(x)}[over]
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, None, mean, rstd, dx, dw, db, scratch)
    torch.cuda.synchronize()
    assert bool(dx[1:rows - 1].isfinite().all()) and bool(dx[0].isnan().all()) and bool(dx[rows - 1].isnan().all())
    for g in (dw, db):
        assert g.isnan().nonzero().flatten().tolist() == [5, cols - 1]


@pytest.mark.parametrize("rows,cols,dtype", [(1100, 1600, "bf16"), (1100, 4096, "bf16"), (600, 8192, "f32"), (600, 13_000, "f32"),
                                             (600, 17_000, "f32")])
def test_backward_parts_of_many_rows(S, rows, cols, dtype):
    """Each gradient alone equals the same gradient of the whole call."""
    log(f"layer norm backward parts {rows}x{cols} {dtype}")
    x, dy = matrix(rows, cols, dtype, 1, 2.0, 0.5), matrix(rows, cols, dtype, 2)
    w = vector(cols, "f32", 3, 0.3, 1.0)
    mean = x.float().mean(1)
    rstd = 1.0 / (x.float().var(1, unbiased=False) + 1e-5).sqrt()
    new = lambda: (torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda"))  # noqa: E731
    whole = new()
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, w, mean, rstd, *whole, scratch)
    for wanted in ((1, 0, 0), (0, 1, 1), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1)):
        part = [t if k else None for t, k in zip(new(), wanted)]
        S.spccl_layer_norm_backward(dy, x, w, mean, rstd, *part, scratch if any(wanted[1:]) else None)
        torch.cuda.synchronize()
        for got, exp in zip(part, whole):
            assert got is None or torch.equal(got, exp), wanted


@pytest.mark.parametrize("cols", [300, 1600, 5000])
def test_many_rows_past_32_bit_offsets(S, cols):
    """Rows whose offsets pass 32 bits in elements and bytes, in the kernel that
    many rows take, also over x."""
    log(f"layer norm backward far rows of many {cols}")
    rows, pitch = 1100, 1 << 21
    buf = torch.empty((rows - 1) * pitch + cols, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, cols), (pitch, 1))
    x.copy_(matrix(rows, cols, "bf16", 3, 2.0, 0.5))
    dy = matrix(rows, cols, "bf16", 4)
    mean = x.float().mean(1)
    rstd = 1.0 / (x.float().var(1, unbiased=False) + 1e-5).sqrt()
    (ex, bx), (ew, bw), (eb, bb) = backward_bounds(dy, x, None, mean, rstd, "bf16")
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    scratch, _ = scratch_for(S, rows, cols)
    S.spccl_layer_norm_backward(dy, x, None, mean, rstd, x, dw, db, scratch)
    torch.cuda.synchronize()
    within(x, ex, bx, "dx")
    within(dw, ew, bw + OUT["f32"] * ew.abs(), "dweight")
    within(db, eb, bb + OUT["f32"] * eb.abs(), "dbias")


@pytest.mark.parametrize("rows,cols,dtype", [(1100, 1600, "bf16"), (1100, 8192, "bf16"), (600, 13_000, "f32"), (3000, 5, "bf16"),
                                             (600, 17_000, "f32")])
def test_backward_of_many_rows_in_a_graph(S, rows, cols, dtype):
    log(f"layer norm backward graph {rows}x{cols} {dtype}")
    x, dy = matrix(rows, cols, dtype, 1, 2.0, 0.5), matrix(rows, cols, dtype, 2)
    w = vector(cols, "f32", 3, 0.3, 1.0)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    new = lambda: (torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda"))  # noqa: E731
    scratch, _ = scratch_for(S, rows, cols)

    def both(o):
        S.spccl_layer_norm(x, w, None, o[0], mean, rstd)
        S.spccl_layer_norm_backward(dy, x, w, mean, rstd, *o, scratch)

    out = new()
    both(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out)
    for k in range(4):
        x.mul_(1.01)
        dy.add_(0.01)
        for t in out:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = new()
        both(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, eager)), k


@pytest.mark.parametrize("cols", [8, 71, 200, 251, 256, 333, 777, 1032, 1111, 1536, 1544, 2056, 3001, 3080, 5000, 6144, 6152, 9999,
                                  10_240, 10_248, 11_111, 12_288, 12_296, 14_001, 20_000, 24_576, 24_584, 30_001])
@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_forward_in_every_layout(S, cols, dtype, wdtype):
    """The widths between the steps of the sizes above; over x too."""
    log(f"layer norm layouts {cols} {dtype} {wdtype}")
    rows = 19
    for pad, offset in ((-cols % 8, 0), (3, 1)):
        x = matrix(rows, cols, dtype, cols, 2.0, 0.7, pad, offset)
        y = matrix(rows, cols, dtype, 1, 1.0, 0.0, pad, offset)
        w, b = vector(cols, wdtype, 2, 0.3, 1.0), vector(cols, wdtype, 3, 0.3, 0.1)
        mean, rstd = torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
        S.spccl_layer_norm(x, w, b, y, mean, rstd, 1e-5)
        torch.cuda.synchronize()
        (m, em), (r, er), (e, ee) = forward_bounds(x, w, b, 1e-5, dtype)
        within(mean[:, None], m, em, "mean")
        within(rstd[:, None], r, er, "rstd")
        within(y, e, ee, "y")
        S.spccl_layer_norm(x, w, b, x, None, None, 1e-5)
        torch.cuda.synchronize()
        assert torch.equal(x, y) and untouched(x) and untouched(y)
