"""Host-side checks of layer norm's entry points: every refusal comes before a
launch, so these run without a GPU."""
import pytest

MB = 1 << 20
OK, INVALID, UNSUPPORTED, WORKSPACE, HIP = 0, 1, 3, 5, 6


@pytest.fixture(scope="module")
def S():
    import paper_2607_04676_amd as S
    return S


def forward(S, x=1 * MB, ldx=100, w=40 * MB, b=41 * MB, y=20 * MB, ldy=100, mean=50 * MB, rstd=51 * MB, rows=10, cols=100,
            dt=0, wdt=0, eps=1e-5):
    return S._lib.spccl_layer_norm(x, ldx, w, b, y, ldy, mean, rstd, rows, cols, dt, wdt, eps, None)


def test_forward_refusals(S):
    assert forward(S, dt=2) == UNSUPPORTED and forward(S, wdt=-1) == UNSUPPORTED
    assert forward(S, cols=1 << 31, ldx=1 << 31, ldy=1 << 31) == UNSUPPORTED and forward(S, rows=1 << 31) == UNSUPPORTED
    assert forward(S, cols=0) == INVALID
    assert forward(S, ldx=99) == INVALID and forward(S, ldy=99) == INVALID
    assert forward(S, eps=-1.0) == INVALID and forward(S, eps=float("nan")) == INVALID
    assert forward(S, x=None) == INVALID and forward(S, y=None) == INVALID
    assert forward(S, x=MB + 2) == INVALID and forward(S, w=40 * MB + 2) == INVALID
    assert forward(S, mean=50 * MB + 2) == INVALID
    assert forward(S, x=None, y=None, rows=0) == OK          # nothing to do


def test_forward_overlaps(S):
    assert forward(S, y=MB + 4) == INVALID                   # one element on
    assert forward(S, y=MB, ldy=101) == INVALID              # x's place at another pitch
    assert forward(S, mean=MB + 400) == INVALID and forward(S, rstd=20 * MB) == INVALID
    assert forward(S, w=20 * MB + 40) == INVALID and forward(S, b=20 * MB) == INVALID
    # column ranges of one buffer interleave without overlapping
    half = dict(ldx=200, ldy=200)
    assert forward(S, y=MB + 4 * 99, **half) == INVALID
    assert forward(S, y=MB + 4 * 101, **half) == INVALID


def backward(S, dy=1 * MB, lddy=100, x=10 * MB, ldx=100, w=40 * MB, mean=50 * MB, rstd=51 * MB, dx=20 * MB, lddx=100,
             dw=60 * MB, db=61 * MB, rows=10, cols=100, dt=0, wdt=0, gdt=0, acc=0, scratch=70 * MB, sb=1 << 30):
    return S._lib.spccl_layer_norm_backward(dy, lddy, x, ldx, w, mean, rstd, dx, lddx, dw, db, rows, cols, dt, wdt, gdt,
                                            acc, scratch, sb, None)


def test_backward_refusals(S):
    assert backward(S, dt=5) == UNSUPPORTED and backward(S, gdt=2) == UNSUPPORTED
    assert backward(S, cols=0) == INVALID and backward(S, lddy=99) == INVALID and backward(S, lddx=99) == INVALID
    assert backward(S, dy=None) == INVALID and backward(S, x=None) == INVALID
    assert backward(S, mean=None) == INVALID and backward(S, rstd=None) == INVALID
    assert backward(S, dw=60 * MB + 1) == INVALID and backward(S, dx=20 * MB + 2) == INVALID
    assert backward(S, scratch=None) == INVALID and backward(S, scratch=70 * MB + 8) == INVALID
    need = S.spccl_layer_norm_scratch_bytes(10, 100)
    assert need > 0 and backward(S, sb=need - 1) == WORKSPACE
    assert backward(S, dx=None, dw=None, db=None) == OK      # nothing wanted


def test_backward_overlaps(S):
    assert backward(S, dx=MB + 4) == INVALID and backward(S, dx=10 * MB + 400) == INVALID
    assert backward(S, dx=50 * MB) == INVALID                # over the statistics
    assert backward(S, dw=20 * MB) == INVALID and backward(S, db=MB) == INVALID
    assert backward(S, db=60 * MB + 4) == INVALID            # the two gradients
    assert backward(S, scratch=20 * MB) == INVALID and backward(S, scratch=60 * MB) == INVALID


def test_scratch_bytes(S):
    f = S.spccl_layer_norm_scratch_bytes
    assert f(0, 100) == 0 and f(10, 0) == 0 and f(1 << 31, 10) == 0
    assert f(1, 1) >= 8
    for cols in (1, 100, 1600, 20_000, 100_000):             # a bounded number of sums per column
        assert f((1 << 31) - 1, cols) <= 8 * cols * 4096


def test_overlaps_of_vectors(S):
    # statistics are written while other rows still read the weight and the bias
    for out in ("mean", "rstd"):
        for read in (40 * MB, 41 * MB):
            assert forward(S, **{out: read}) == INVALID
            assert forward(S, **{out: read + 396}) == INVALID
            assert forward(S, **{out: read - 36}) == INVALID
    assert forward(S, mean=50 * MB, rstd=50 * MB + 36) == INVALID
    # and the sums of the columns while others read the weight and the statistics
    for out in ("dw", "db", "scratch"):
        for read, size in ((40 * MB, 400), (50 * MB, 40), (51 * MB, 40)):
            assert backward(S, **{out: read}) == INVALID
            if out != "scratch":
                assert backward(S, **{out: read + size - 4}) == INVALID
                assert backward(S, **{out: read - 396}) == INVALID
    assert backward(S, scratch=61 * MB) == INVALID


def test_columns_that_a_grid_cannot_take(S):
    # the reduction of the weight's gradient takes 1024 threads for 32 columns, of fewer than 2^32
    for cols in (1 << 26, (1 << 27) - 1):
        wide = dict(cols=cols, rows=0)
        assert forward(S, ldx=cols, ldy=cols, **wide) == UNSUPPORTED
        assert backward(S, ldx=cols, lddy=cols, lddx=cols, **wide) == UNSUPPORTED
        assert S.spccl_layer_norm_scratch_bytes(10, cols) == 0
    cols = (1 << 26) - 1
    assert forward(S, cols=cols, rows=0, ldx=cols, ldy=cols) == OK
    assert backward(S, cols=cols, rows=0, ldx=cols, lddy=cols, lddx=cols, dw=None, db=None) == OK
    assert S.spccl_layer_norm_scratch_bytes(10, cols) == 8 * cols
