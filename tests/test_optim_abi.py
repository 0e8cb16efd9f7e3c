"""Host-side checks of the pruning's and AdamW's entry points: every refusal
comes before a launch, so these run without a GPU."""
import ctypes

import pytest

MB = 1 << 20
OK, INVALID, CAPACITY, UNSUPPORTED, WORKSPACE, HIP = 0, 1, 2, 3, 5, 6


@pytest.fixture(scope="module")
def S():
    import paper_2607_04676_amd as S
    return S


def prune(S, grad=1 * MB, res=10 * MB, tau=20 * MB, leak=1.0, out=30 * MB, n=1000, dt=0):
    return S._lib.spccl_prune(grad, res, tau, leak, out, n, dt, None)


def test_prune_refusals(S):
    assert prune(S, dt=2) == UNSUPPORTED and prune(S, n=1 << 40) == UNSUPPORTED
    assert prune(S, leak=-0.1) == INVALID and prune(S, leak=1.1) == INVALID and prune(S, leak=float("nan")) == INVALID
    assert prune(S, tau=None) == INVALID and prune(S, tau=20 * MB + 2) == INVALID
    for bad in (dict(grad=None), dict(res=None), dict(out=None), dict(grad=MB + 2), dict(res=10 * MB + 2),
                dict(out=30 * MB + 1)):
        assert prune(S, **bad) == INVALID, bad
    assert prune(S, out=MB + 4) == INVALID and prune(S, res=MB) == INVALID and prune(S, res=30 * MB + 400) == INVALID
    assert prune(S, tau=30 * MB + 40) == INVALID and prune(S, tau=10 * MB) == INVALID
    assert prune(S, n=0, grad=None, res=None, out=None) == OK


def tensor(S, **kw):
    d = dict(param=1 * MB, model=None, grad=S.spccl_operand_t(S.SPCCL_ARRAY, 0, 2 * MB, 4000), grad_offset=0, grad_n=0,
             m=3 * MB, v=4 * MB, m_scale=None, v_scale=None, n=1000, weight_decay=0.0)
    d.update(kw)
    return S.spccl_adamw_tensor_t(**d)


def plan(S, tensors, pdt=0, gdt=0, state=0, table=100 * MB, size=MB, out=None):
    arr = (S.spccl_adamw_tensor_t * len(tensors))(*tensors)
    p = S.spccl_adamw_plan_t() if out is None else out
    return S._lib.spccl_adamw_plan(arr, len(tensors), pdt, gdt, state, table, size, ctypes.byref(p), None)


def stream(S, fmt=1, ptr=2 * MB, size=MB):
    return S.spccl_operand_t(S.SPCCL_STREAM, fmt, ptr, size)


def test_plan_refusals(S):
    t = lambda **kw: [tensor(S, **kw)]  # noqa: E731
    assert plan(S, t(), pdt=2) == UNSUPPORTED and plan(S, t(), gdt=5) == UNSUPPORTED and plan(S, t(), state=2) == UNSUPPORTED
    assert plan(S, t(n=1 << 32)) == UNSUPPORTED
    assert plan(S, t(weight_decay=-1.0)) == INVALID and plan(S, t(weight_decay=float("nan"))) == INVALID
    for bad in (dict(param=None), dict(m=None), dict(v=None), dict(param=MB + 2), dict(m=3 * MB + 1), dict(v=4 * MB + 2),
                dict(model=50 * MB + 1), dict(m_scale=60 * MB), dict(v_scale=61 * MB)):
        assert plan(S, t(**bad)) == INVALID, bad
    assert plan(S, t(grad=S.spccl_operand_t(S.SPCCL_ARRAY, 0, None, 4000))) == INVALID
    assert plan(S, t(grad=S.spccl_operand_t(S.SPCCL_ARRAY, 0, 2 * MB + 2, 4000))) == INVALID
    assert plan(S, t(grad=S.spccl_operand_t(S.SPCCL_ARRAY, 0, 2 * MB, 3999))) == CAPACITY
    assert plan(S, t(grad=S.spccl_operand_t(7, 0, 2 * MB, 4000))) == INVALID
    assert plan(S, t(model=50 * MB), pdt=1) == INVALID           # a copy of a bf16 parameter
    assert plan(S, t(), state=1) == INVALID                      # 8 bits without scales
    assert plan(S, t(), size=0) == WORKSPACE and plan(S, t(), table=None) == INVALID and plan(S, t(), table=MB + 8) == INVALID
    arr = (S.spccl_adamw_tensor_t * 1)(tensor(S))
    assert S._lib.spccl_adamw_plan(arr, 1, 0, 0, 0, 100 * MB, MB, None, None) == INVALID
    assert S._lib.spccl_adamw_plan(None, 1, 0, 0, 0, 100 * MB, MB, None, None) == INVALID
    assert S._lib.spccl_adamw_plan(arr, -1, 0, 0, 0, 100 * MB, MB, None, None) == INVALID


def test_stream_refusals(S):
    t = lambda **kw: [tensor(S, **{**dict(grad=stream(S), grad_n=4096), **kw})]  # noqa: E731
    assert plan(S, t(grad=stream(S, fmt=2))) == UNSUPPORTED      # COO
    assert plan(S, t(grad=stream(S, fmt=9))) == INVALID
    assert plan(S, t(grad=stream(S, ptr=2 * MB + 8))) == INVALID
    assert plan(S, t(grad=stream(S, size=47))) == CAPACITY
    assert plan(S, t(grad_offset=32)) == INVALID
    assert plan(S, t(grad_offset=3136)) == INVALID               # its last elements past the message
    assert plan(S, t(grad_offset=8192)) == INVALID
    assert plan(S, t(grad_n=999)) == INVALID and plan(S, t(grad_n=1 << 32)) == UNSUPPORTED


def test_overlaps(S):
    two = lambda **kw: [tensor(S), tensor(S, **{**dict(param=11 * MB, m=13 * MB, v=14 * MB), **kw})]  # noqa: E731
    for bad in (dict(param=MB + 3996), dict(m=MB), dict(v=3 * MB + 400), dict(model=4 * MB), dict(param=2 * MB + 40),
                dict(param=100 * MB), dict(m=11 * MB), dict(v=13 * MB + 3996),
                dict(grad=S.spccl_operand_t(S.SPCCL_ARRAY, 0, 3 * MB + 4, 4000))):
        assert plan(S, two(**bad)) == INVALID, bad
    # a shared gradient is fine: the call gets as far as its first launch
    p = S.spccl_adamw_plan_t()
    assert plan(S, two(), out=p) in (OK, HIP)


def test_plan_bytes(S):
    f = lambda ts: S._lib.spccl_adamw_plan_bytes((S.spccl_adamw_tensor_t * len(ts))(*ts), len(ts))  # noqa: E731
    assert S._lib.spccl_adamw_plan_bytes(None, 3) == 0 and S._lib.spccl_adamw_plan_bytes(None, -1) == 0
    assert f([tensor(S)]) >= 128 + 4
    assert f([tensor(S, n=0)]) < f([tensor(S)]) + 1
    assert f([tensor(S, n=1 << 31)]) >= 128 + 4 * ((1 << 31) // 4096)


def test_step_refusals(S):
    p = S.spccl_adamw_plan_t()
    h = S.spccl_adamw_t(1e-3, 0.9, 0.999, 1e-8, 1, 0)
    step = lambda plan=p, hyper=h, scale=None, ws=MB, wsb=256: S._lib.spccl_adamw_step(  # noqa: E731
        None if plan is None else ctypes.byref(plan), None if hyper is None else ctypes.byref(hyper), scale, ws, wsb, None)
    assert step() == INVALID                                     # not a plan
    empty = S.spccl_adamw_plan_t()
    assert S._lib.spccl_adamw_plan(None, 0, 0, 0, 0, None, 0, ctypes.byref(empty), None) == OK
    assert step(empty) == OK                                     # no tensors: nothing to launch
    assert step(None) == INVALID and step(empty, None) == INVALID
    assert step(empty, ws=None) == INVALID and step(empty, ws=MB + 8) == INVALID and step(empty, wsb=255) == WORKSPACE
    assert step(empty, scale=MB + 2) == INVALID
    nan = float("nan")
    for bad in (dict(lr=-1.0), dict(lr=nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan),
                dict(eps=-1e-8), dict(eps=nan), dict(step=0)):
        d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0)
        d.update(bad)
        assert step(empty, S.spccl_adamw_t(**d)) == INVALID, bad


def test_values_in_host_memory(S):
    """A threshold or a scale that kernels could not read is refused by the
    binding, before the call."""
    torch = pytest.importorskip("torch")
    x, value = torch.zeros(8), torch.tensor([0.5])
    with pytest.raises(ValueError, match="threshold"):
        S.spccl_prune(x, x.clone(), value, 1.0, x.clone())
    with pytest.raises(ValueError, match="grad_scale"):
        S.spccl_adamw_step(S.spccl_adamw_plan_t(), torch.zeros(256, dtype=torch.uint8), 1e-3, grad_scale=value)
