"""The AdamW step over many tensors.

Moments are defined operation by operation in fp32, so they are compared bit
for bit with a numpy computation of the same operations, and 8-bit moments with
an integer implementation of their format.  Everything is also held against
the formula in 64 bits, with u = 2^-24: a moment is a sum of two products whose
factors are rounded constants, within 4 u of its terms (a second moment's g^2
adds 2 u more); an update m / (sqrt(v) c + eps) * rate is within 12 u of itself
beyond what its moments bring (sqrt halves v's), and param (1 - lr wd) within
3 u.
"""
import ctypes

import numpy as np
import pytest

from helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
f32 = np.float32
SIZES = [1, 2, 3, 5, 0, 31, 32, 33, 63, 64, 65, 100, 4095, 4096, 4097, 8200, 70_001]
BLOCK = 32


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_04676_amd as S
    return S


# ---- the format of 8-bit moments, in integers ------------------------------------------

def mix(x):
    x = np.asarray(x, np.uint64) & 0xFFFFFFFF
    for shift, mul in ((16, 0x9E3779B1), (15, 0x6A09E667)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(mul)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(count, counter, seed, second=False):
    key = mix(mix(seed & 0xFFFFFFFF) ^ np.uint64(seed >> 32))
    at = np.arange(count, dtype=np.uint64) + np.uint64(counter)
    h = mix((at >> np.uint64(2)) ^ key)
    if second:
        h = (h * np.uint64(0x6A09E667)) & np.uint64(0xFFFFFFFF)
    return (h + (at & np.uint64(3)) * np.uint64(0x9E3779B9)) & np.uint64(0xFFFFFFFF)


def e4m3_table():
    code = np.arange(256)
    e, man = (code >> 3) & 15, code & 7
    value = np.where(e == 0, man * 2.0 ** -9, (8 + man) * 2.0 ** (e - 10.0))
    value[(e == 15) & (man == 7)] = np.nan
    return np.where(code >> 7, -value, value)


E4M3 = e4m3_table()


def decode(code, scale):
    n = code.size
    with np.errstate(invalid="ignore"):
        s = np.where(scale == 255, np.inf, np.where(scale == 0, 0.0, 2.0 ** (scale.astype(np.float64) - 127)))
        return (E4M3[code] * np.repeat(s, BLOCK)[:n]).astype(f32)


def encode(x, r, second):
    """Codes and scales of fp32 moments with 32 random bits each."""
    n = x.size
    blocks = -(-n // BLOCK)
    a = np.zeros(blocks * BLOCK, f32)
    a[:n] = np.abs(x)
    top = a.view(np.uint32).reshape(blocks, BLOCK).max(1) >> 23
    scale = np.where(top == 255, 255, np.maximum(top, 32) - 7)
    lost = np.repeat(top == 255, BLOCK)[:n]
    y = a[:n].astype(np.float64) / np.repeat(2.0 ** (np.where(top == 255, 127, scale).astype(np.float64) - 127), BLOCK)[:n]
    bits = (r & np.uint64(0xFFFFF)) if second else (r >> np.uint64(12))
    with np.errstate(invalid="ignore"):
        if second:
            y = np.where(a[:n] > 0, np.maximum(y, 2.0 ** -9), y)
        y[lost] = 0.0
        e = np.floor(np.log2(np.maximum(y, 2.0 ** -6)))
        unit = 2.0 ** (np.maximum(e, -6) - 3)                    # the grid around y
        # y in units of 2^-20 of the grid, as fp32 holds it: below the normal
        # codes it is first rounded at 2^-29, to even
        fine = np.where(y < 2.0 ** -6, np.rint(y * 2.0 ** 29), y / unit * 2.0 ** 20)
        steps = np.floor((np.floor(fine) + bits.astype(np.float64)) / 2.0 ** 20)
        value = steps * unit
    code = np.searchsorted(E4M3[:127], value)
    assert np.array_equal(E4M3[code], value)
    code = code | np.where(np.signbit(x), 128, 0)
    return code.astype(np.uint8), scale.astype(np.uint8), lost


# ---- a plan and its reference ----------------------------------------------------------

class Case:
    """Tensors of the given sizes, each a view inside a larger buffer whose other
    elements must stay, and the same in numpy."""

    def __init__(self, S, sizes, pdtype, gdtype, state, form, seed, copy=False, shift=0, scale=1e-3, decay=(0.1, 0.0)):
        self.S, self.sizes, self.state, self.pdtype, self.gdtype = S, sizes, state, pdtype, gdtype
        rng = np.random.default_rng(seed)
        self.starts, at = [], 0
        for n in sizes:
            self.starts.append(at)
            at += -(-n // 64) * 64
        self.total = at
        self.decay = [decay[i % len(decay)] for i in range(len(sizes))]
        self.copy = copy

        def buffer(values, dtype):
            t = torch.full((self.total + shift + 8,), -99.0, dtype=torch.float32).to(dtype)
            t[shift:shift + self.total] = torch.from_numpy(values).to(dtype)
            return t.cuda()
        pick = lambda t: [t[shift + s:shift + s + n] for s, n in zip(self.starts, sizes)]  # noqa: E731
        self.buffers = {"param": buffer(rng.normal(0, 0.02, self.total).astype(f32), DT[pdtype])}
        if copy:
            self.buffers["model"] = buffer(np.zeros(self.total, f32), torch.bfloat16)
        grad = rng.normal(0, scale, self.total).astype(f32)
        self.used = np.zeros(self.total, bool)
        for s, n in zip(self.starts, sizes):
            self.used[s:s + n] = True
        if form != "array":
            grad[(rng.random(self.total) < 0.9) & (np.arange(self.total) // 4096 % 3 != 1)] = 0      # some tiles full
            grad[~self.used] = 0
        self.grad_buffer = buffer(grad, DT[gdtype])
        self.grad = self.grad_buffer[shift:shift + self.total].float().cpu().numpy()
        self.form = form
        m0 = rng.normal(0, 3 * scale / 10, self.total).astype(f32)
        v0 = (np.square(rng.normal(0, scale, self.total)) + 1e-12).astype(f32)
        if state == 8:
            r = random_bits(self.total, 0, seed)
            for k, x in (("m", m0), ("v", v0)):
                x[~self.used] = 0
                code, scales, _ = encode(x, r, k == "v")
                c = torch.full((self.total + shift + 8,), 0x55, dtype=torch.uint8)
                c[shift:shift + self.total] = torch.from_numpy(code)
                self.buffers[k] = c.cuda()
                self.buffers[k + "_scale"] = torch.from_numpy(np.concatenate([scales, np.full(8, 77, np.uint8)])).cuda()
        else:
            self.buffers["m"], self.buffers["v"] = buffer(m0, torch.float32), buffer(v0, torch.float32)
        self.shift = shift
        self.views = {k: pick(t) for k, t in self.buffers.items() if not k.endswith("_scale")}
        for k in ("m_scale", "v_scale"):
            if k in self.buffers:
                self.views[k] = [self.buffers[k][s // BLOCK:s // BLOCK + -(-n // BLOCK)] for s, n in zip(self.starts, sizes)]
        self.message()
        tensors = []
        for i, n in enumerate(sizes):
            kw = {k: self.views[k][i] for k in ("m", "v", "m_scale", "v_scale", "model") if k in self.views}
            stream = form in ("pici", "dense") or (form == "mixed" and i % 2)
            if stream:
                fmt = S.SPCCL_FMT_DENSE if form == "dense" else S.SPCCL_FMT_PICI
                kw.update(grad=S.operand(self.msg, S.SPCCL_STREAM, fmt), grad_offset=self.starts[i], grad_n=self.total,
                          grad_dtype=S.SPCCL_F32 if gdtype == "f32" else S.SPCCL_BF16)
            else:
                kw["grad"] = self.grad_buffer[shift + self.starts[i]:shift + self.starts[i] + n]
            tensors.append(S.adamw_tensor(self.views["param"][i], weight_decay=self.decay[i], **kw))
        self.tensors = tensors
        self.ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
        table = torch.full((S.spccl_adamw_plan_bytes(tensors) + 64,), 0xEE, dtype=torch.uint8, device="cuda")
        self.plan = S.spccl_adamw_plan(tensors, table[:-64])
        torch.cuda.synchronize()
        assert bool((table[-64:] == 0xEE).all())

    def message(self):
        S = self.S
        if self.form == "array":
            return
        dt = S.SPCCL_F32 if self.gdtype == "f32" else S.SPCCL_BF16
        src = self.grad_buffer[self.shift:self.shift + self.total]
        self.msg = S.alloc_stream(self.total, dt)
        if self.form == "dense":
            S.spccl_encode_dense(src, self.msg)
        else:
            ws = S.alloc_workspace(self.total, dt)
            S.spccl_compress(src, self.msg, ws)
            torch.cuda.synchronize()
            assert S.spccl_read_status(ws) == 0

    def read(self):
        """Each tensor's arrays in numpy: params and moments in fp32, codes as bytes."""
        out = []
        for i in range(len(self.sizes)):
            d = {}
            for k, v in self.views.items():
                t = v[i]
                d[k] = t.cpu().numpy() if t.dtype in (torch.uint8, torch.float32) else t.float().cpu().numpy()
            out.append(d)
        return out

    def expect(self, before, hyper, seed, grad_scale):
        """The moments as they have to be, bit for bit, and the parameters in 64
        bits with their bounds."""
        lr, b1, b2, eps, t = hyper
        exp, counter = [], 0
        for i, (n, s) in enumerate(zip(self.sizes, self.starts)):
            b = before[i]
            g = self.grad[s:s + n] * f32(grad_scale)
            m0, v0 = (decode(b["m"], b["m_scale"]), decode(b["v"], b["v_scale"])) if self.state == 8 else (b["m"], b["v"])
            with np.errstate(over="ignore", invalid="ignore", under="ignore"):
                m = m0 * f32(b1) + g * f32(1.0 - b1)
                v = v0 * f32(b2) + (g * g) * f32(1.0 - b2)
            e = {"m32": m, "v32": v}
            if self.state == 8:
                r = random_bits(n, counter, seed)
                e["m"], e["m_scale"], e["lost"] = encode(m, r, False)
                e["v"], e["v_scale"], lost = encode(v, r, True)
                e["lost_v"] = lost
            g64 = self.grad[s:s + n].astype(np.float64) * float(f32(grad_scale))
            m0, v0 = m0.astype(np.float64), v0.astype(np.float64)
            with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
                m64, v64 = b1 * m0 + (1 - b1) * g64, b2 * v0 + (1 - b2) * g64 * g64
                em = 6 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * g64)) + 2e-45
                ev = 8 * U * v64 + 2e-45
                denom = np.sqrt(v64 / (1 - b2 ** t)) + eps
                # sqrt(v) moves by at most ev / (2 sqrt(v)) or sqrt(ev)
                ed = np.minimum(ev / (2 * np.sqrt(np.maximum(v64, 1e-300))), np.sqrt(ev)) / np.sqrt(1 - b2 ** t)
                up = lr * (m64 / (1 - b1 ** t)) / denom
                low = denom - ed
                eu = np.where(low > denom / 2, lr / (1 - b1 ** t) * em / np.maximum(low, 1e-300)
                              + np.abs(up) * (2 * ed / denom + 16 * U), np.inf)
                p0 = b["param"].astype(np.float64)
                keep = 1 - lr * self.decay[i]
                e["param"] = p0 * keep - up
                e["bound"] = eu + 4 * U * np.abs(p0) + 2 * U * np.abs(up) + 1e-44
                e["m64"], e["em"], e["v64"], e["ev"] = m64, em, v64, ev
            exp.append(e)
            counter += -(-n // 64) * 64
        return exp

    def check(self, got, exp):
        for i, n in enumerate(self.sizes):
            g, e = got[i], exp[i]
            what = f"tensor {i} of {n}"
            if self.state == 8:
                assert np.array_equal(g["m_scale"], e["m_scale"]), what
                assert np.array_equal(g["v_scale"], e["v_scale"]), what
                ok = ~e["lost"]
                assert np.array_equal(g["m"][ok], e["m"][ok]), what
                assert np.isnan(decode(g["m"], g["m_scale"])[~ok]).all(), what
                ok = ~e["lost_v"]
                assert np.array_equal(g["v"][ok], e["v"][ok]), what
                assert np.isnan(decode(g["v"], g["v_scale"])[~ok]).all(), what
            else:
                nan = np.isnan(e["m32"])
                assert np.array_equal(g["m"].view(np.uint32)[~nan], e["m32"].view(np.uint32)[~nan]), what
                assert np.isnan(g["m"][nan]).all()
                nan = np.isnan(e["v32"])
                assert np.array_equal(g["v"].view(np.uint32)[~nan], e["v32"].view(np.uint32)[~nan]), what
                fine = np.isfinite(e["m64"]) & np.isfinite(g["m"]) & np.isfinite(g["v"])
                assert (np.abs(g["m"] - e["m64"])[fine] <= e["em"][fine]).all(), what
                assert (np.abs(g["v"] - e["v64"])[fine] <= e["ev"][fine]).all(), what
            fine = np.isfinite(e["param"])
            bound = e["bound"] + (2.0 ** -7 * np.abs(e["param"]) + 1e-38 if self.pdtype == "bf16" else 0.0)
            err = np.abs(g["param"].astype(np.float64) - e["param"])
            assert (err[fine] <= bound[fine]).all(), f"{what}: {np.nanmax(err[fine] / bound[fine])} times the bound"
            if self.copy:
                exp_copy = torch.from_numpy(g["param"]).to(torch.bfloat16).float().numpy()
                assert np.array_equal(g["model"].view(np.uint32), exp_copy.view(np.uint32)), what
        for k, t in self.buffers.items():      # what lies between and around the tensors
            if k.endswith("_scale"):
                assert bool((t[-8:] == 77).all())
                continue
            outside = torch.ones(t.numel(), dtype=torch.bool)
            for s, n in zip(self.starts, self.sizes):
                outside[self.shift + s:self.shift + s + n] = False
            assert torch.equal(t[outside.cuda()], self.untouched[k][outside.cuda()]), k

    def step(self, hyper, seed, grad_scale=None, stream=None):
        self.untouched = {k: t.clone() for k, t in self.buffers.items()}
        lr, b1, b2, eps, t = hyper
        self.S.spccl_adamw_step(self.plan, self.ws, lr, b1, b2, eps, t, seed, grad_scale, stream)
        torch.cuda.synchronize()


HYPER = (3e-4, 0.9, 0.999, 1e-8, 7)


@pytest.mark.parametrize("form", ["array", "pici", "dense", "mixed"])
@pytest.mark.parametrize("gdtype", ["f32", "bf16"])
@pytest.mark.parametrize("pdtype,copy,shift", [("f32", False, 0), ("f32", True, 1), ("bf16", False, 3)])
@pytest.mark.parametrize("state", [32, 8])
def test_step(S, state, pdtype, copy, shift, gdtype, form):
    log(f"adamw {state} {pdtype} {gdtype} {form} copy={copy} shift={shift}")
    c = Case(S, SIZES, pdtype, gdtype, state, form, 1, copy, shift)
    scale = torch.tensor([0.37], device="cuda")
    for t in range(3):                                          # three steps, each from what the last one left
        before = c.read()
        hyper = (HYPER[0], 0.9, 0.95, 1e-8, 1 + 400 * t)
        seed = (0x123456789ABCDEF * (t + 1)) % (1 << 64)
        c.step(hyper, seed, scale if t else None)
        c.check(c.read(), c.expect(before, hyper, seed, f32(0.37) if t else 1.0))
    assert S.spccl_read_status(c.ws) == 0


@pytest.mark.parametrize("state", [32, 8])
@pytest.mark.parametrize("hyper", [(0.0, 0.9, 0.999, 1e-8, 1), (1e-2, 0.0, 0.0, 1e-6, 1), (1e-3, 0.5, 0.99, 1e-8, 1 << 40)])
def test_hyper_parameters(S, state, hyper):
    log(f"adamw hyper {hyper} {state}")
    c = Case(S, [1000, 77], "f32", "f32", state, "array", 2)
    before = c.read()
    c.step(hyper, 5)
    c.check(c.read(), c.expect(before, hyper, 5, 1.0))


@pytest.mark.parametrize("state", [32, 8])
@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1e-9, 1.0, 1e9, 1e15])
def test_magnitudes(S, state, scale):
    """Gradients whose squares leave the normal numbers on either side of the
    usual, down to underflow."""
    log(f"adamw magnitudes {scale} {state}")
    c = Case(S, [5000], "f32", "f32", state, "array", 3, scale=scale)
    before = c.read()
    c.step(HYPER, 9)
    c.check(c.read(), c.expect(before, HYPER, 9, 1.0))


@pytest.mark.parametrize("state", [32, 8])
def test_from_zero_and_without_gradient(S, state):
    """Zeroed moments; then no gradient at all: moments decay and parameters move."""
    log(f"adamw zero {state}")
    c = Case(S, [300, 4096], "f32", "f32", state, "array", 4)
    for k in ("m", "v", "m_scale", "v_scale"):
        if k in c.buffers:
            for t in c.views[k]:
                t.zero_()
    before = c.read()
    c.step((1e-3, 0.9, 0.999, 1e-8, 1), 3)
    c.check(c.read(), c.expect(before, (1e-3, 0.9, 0.999, 1e-8, 1), 3, 1.0))
    c.grad_buffer.zero_()
    c.grad[:] = 0
    before = c.read()
    c.step((1e-3, 0.9, 0.999, 1e-8, 2), 4)
    c.check(c.read(), c.expect(before, (1e-3, 0.9, 0.999, 1e-8, 2), 4, 1.0))


@pytest.mark.parametrize("state", [32, 8])
def test_not_finite_stays_where_it_is(S, state):
    """A NaN or infinite gradient spoils its element's moments; with 8-bit
    moments its block's, whose scale says so.  No other element changes its course."""
    log(f"adamw nan {state}")
    c = Case(S, [1000, 200], "f32", "f32", state, "array", 5)
    clean = Case(S, [1000, 200], "f32", "f32", state, "array", 5)
    for i, x in ((0, np.nan), (333, np.inf), (999, -np.inf)):
        c.grad_buffer[i] = float(x)
        c.grad[i] = x
    before = c.read()
    c.step(HYPER, 6)
    clean.step(HYPER, 6)
    got, ref = c.read(), clean.read()
    c.check(got, c.expect(before, HYPER, 6, 1.0))
    other = np.ones(1000, bool)
    other[[0, 333, 999]] = False
    assert np.array_equal(got[0]["param"][other], ref[0]["param"][other])
    assert np.array_equal(got[1]["param"], ref[1]["param"])
    if state == 8:
        assert got[0]["m_scale"][[0, 10, 31]].tolist() == [255] * 3 and (got[0]["m_scale"] == 255).sum() == 3
        # the next step keeps it
        c.grad_buffer[:1200].fill_(1e-3)
        c.step(HYPER, 7)
        assert (c.read()[0]["v_scale"] == 255).sum() == 3


def test_stochastic_rounding_is_even(S):
    """Equal moments in every element, many seeds: the mean stored value is the
    moment.  A stored value is one of two neighbours a distance q apart, so the
    mean of N has a deviation of at most q / 2 / sqrt(N); 6 of them, and the
    resolution of the random bits (2^-20 q), are allowed."""
    log("adamw rounding")
    n, seeds = 1 << 16, 8
    for m0, g0 in ((0.0, 1.17e-3), (0.0, -3.3e-7), (0.0, 0.71)):
        sums, count = np.zeros(2), 0
        for seed in range(seeds):
            c = Case(S, [n], "f32", "f32", 8, "array", 1)
            for k in ("m", "v", "m_scale", "v_scale"):
                c.views[k][0].zero_()
            c.grad_buffer.fill_(g0)
            # one element a block is larger, so that the others lie lower in its range
            c.views["param"][0].zero_()
            c.grad_buffer[:n].view(-1, 32)[:, 0] = 20 * g0
            c.step((1e-3, 0.9, 0.999, 1e-8, 1), seed * 0x1234567 + (seed << 40))
            got = c.read()[0]
            keep = np.arange(n) % 32 != 0
            for k in (0, 1):
                sums[k] += decode(got["mv"[k]], got["mv"[k] + "_scale"]).astype(np.float64)[keep].sum()
            count += keep.sum()
        g = f32(g0)
        for k, x in ((0, g * f32(1.0 - 0.9)), (1, (g * g) * f32(1.0 - 0.999))):
            top = np.floor(np.log2(abs(float(x)) * (20 if k == 0 else 400)))
            q = max(2.0 ** (np.floor(np.log2(abs(float(x)))) - 3), 2.0 ** (top - 7 - 9))
            tol = 6 * q / 2 / np.sqrt(count) + 2.0 ** -20 * q + 4 * U * abs(float(x))
            assert abs(sums[k] / count - float(x)) <= tol, (g0, k)


def test_sixteen_bit_parameters_are_rounded_evenly(S):
    """bf16 parameters: updates far below half a unit still move the mean.  The
    mean of N is within 6 q / 2 / sqrt(N) + 2^-16 q of the exact parameter."""
    log("adamw bf16 rounding")
    n, seeds, total, count = 1 << 16, 8, 0.0, 0
    hyper = (1e-4, 0.0, 0.0, 1e-8, 1)                           # update = lr * sign(g)
    for seed in range(seeds):
        c = Case(S, [n], "bf16", "f32", 32, "array", 1, decay=(0.0,))
        c.views["param"][0].fill_(1.0)
        c.grad_buffer.fill_(0.5)
        c.step(hyper, seed * 7 + 1)
        total += c.read()[0]["param"].astype(np.float64).sum()
        count += n
    q = 2.0 ** -8                                               # below 1
    assert abs(total / count - (1.0 - 1e-4)) <= 6 * q / 2 / np.sqrt(count) + 2.0 ** -16 * q + 16 * U


def test_a_second_moment_stays_above_zero(S):
    log("adamw floor")
    c = Case(S, [64], "f32", "f32", 8, "array", 1)
    g = np.full(64, 1e-8, f32)
    g[0] = 1.0                                                  # 16 decades above the others' squares
    c.grad_buffer[:64] = torch.from_numpy(g).cuda()
    c.grad[:64] = g
    for seed in range(10):
        for k in ("m", "v", "m_scale", "v_scale"):
            c.views[k][0].zero_()
        c.step((1e-3, 0.9, 0.999, 1e-8, 1), seed)
        assert (c.read()[0]["v"] > 0).all()


def test_many_tensors(S):
    """More tensors than one batch of the table, and a few of no elements."""
    log("adamw many tensors")
    sizes = [(i * 37) % 130 for i in range(1500)]
    for state in (32, 8):
        c = Case(S, sizes, "f32", "bf16", state, "mixed", 6)
        before = c.read()
        c.step(HYPER, 11)
        c.check(c.read(), c.expect(before, HYPER, 11, 1.0))


def test_no_tensors(S):
    table = torch.empty(16, dtype=torch.uint8, device="cuda")
    plan = S.spccl_adamw_plan([], table)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    S.spccl_adamw_step(plan, ws, 1e-3)
    torch.cuda.synchronize()


def test_past_32_bit_offsets(S):
    """A tensor of 2^30 + 5 elements: its fp32 arrays pass 4 GiB."""
    log("adamw large")
    n = (1 << 30) + 5
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    state = S.alloc_adamw_state(n)
    at = torch.tensor([0, (1 << 29) - 1, 1 << 29, (1 << 30) - 1, 1 << 30, n - 1], device="cuda")
    g[at] = 1.0
    tensors = [S.adamw_tensor(p, g, **state)]
    plan = S.spccl_adamw_plan(tensors, torch.empty(S.spccl_adamw_plan_bytes(tensors), dtype=torch.uint8, device="cuda"))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    S.spccl_adamw_step(plan, ws, 0.5, 0.0, 0.0, 0.0, 1)          # 0 / 0 where there is no gradient
    torch.cuda.synchronize()
    assert bool((p[at] == -0.5).all())
    assert int(p.isnan().sum()) == n - at.numel()
    assert bool((state["m"][at] == 1.0).all()) and int(torch.count_nonzero(state["v"])) == at.numel()


def test_corrupt_messages(S):
    """A message that fails its header checks changes nothing and says so; a tile
    whose words and index disagree counts as empty."""
    log("adamw corrupt")
    for byte, value in ((0, 0), (4, 9), (6, 1), (8, 1), (16, 255), (40, 1)):
        c = Case(S, [3000, 9000], "f32", "f32", 32, "pici", 7)
        c.msg[byte] += value + (byte == 0)
        before = c.read()
        c.step(HYPER, 1)
        after = c.read()
        assert S.spccl_read_status(c.ws) == 4, byte
        for b, a in zip(before, after):
            assert all(np.array_equal(b[k].view(np.uint8), a[k].view(np.uint8)) for k in b), byte
    for where in ("word", "index", "end"):
        c = Case(S, [3000, 9000], "f32", "f32", 32, "pici", 8)
        n = c.total
        tiles = -(-n // 4096)
        index = c.msg[48 + 512 * tiles:48 + 512 * tiles + 4 * (tiles + 1)].view(torch.int32)
        if where == "word":
            c.msg[48 + 512 + 3] ^= 0x10                          # tile 1: one bit more or fewer
            bad = [1]
        elif where == "index":
            index[2] += 1                                        # tiles 1 and 2
            bad = [1, 2]
        else:
            last = c.msg[48 + 512 * (tiles - 1):48 + 512 * tiles].view(torch.int64)
            last[63] |= -(1 << 63)                               # a row past the end
            bad = [tiles - 1]
        for b in bad:
            c.grad[b * 4096:(b + 1) * 4096] = 0
        before = c.read()
        c.step(HYPER, 1)
        c.check(c.read(), c.expect(before, HYPER, 1, 1.0))
        assert S.spccl_read_status(c.ws) == 4, where


def test_a_message_of_another_size_or_type(S):
    log("adamw other message")
    c = Case(S, [3000], "f32", "f32", 32, "pici", 7)
    for other in (torch.zeros(2000, device="cuda"), torch.zeros(c.total, dtype=torch.bfloat16, device="cuda")):
        dt = S.SPCCL_F32 if other.dtype == torch.float32 else S.SPCCL_BF16
        ws = S.alloc_workspace(4096, dt)
        S.spccl_compress(other, c.msg, ws) if other.numel() * 4 < c.msg.numel() and dt == S.SPCCL_F32 and \
            S.spccl_stream_bound(other.numel(), dt) <= c.msg.numel() else S.spccl_encode_dense(other, c.msg)
        before = c.read()
        c.step(HYPER, 1)
        assert S.spccl_read_status(c.ws) == 4
        assert np.array_equal(before[0]["param"], c.read()[0]["param"])


def test_on_another_stream_and_in_a_graph(S):
    log("adamw graph")
    for state in (32, 8):
        for form in ("array", "pici"):
            c, e = (Case(S, [5000, 64, 4097], "f32", "f32", state, form, 9) for _ in range(2))
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            c.step(HYPER, 21, stream=side)
            e.step(HYPER, 21)
            graph = torch.cuda.CUDAGraph()
            lr, b1, b2, eps, t = HYPER
            with torch.cuda.graph(graph):
                S.spccl_adamw_step(c.plan, c.ws, lr, b1, b2, eps, t, 22)
            for k in range(4):
                for x in (c, e):
                    x.grad_buffer.mul_(1.1)
                    x.message()
                if form == "pici":                               # both plans keep their message's place
                    c.tensors[0]._tensors[1]._tensor.copy_(c.msg)
                    e.tensors[0]._tensors[1]._tensor.copy_(e.msg)
                graph.replay()
                torch.cuda.synchronize()
                e.step(HYPER, 22)
                for a, b in zip(c.read(), e.read()):
                    assert all(np.array_equal(a[q].view(np.uint8), b[q].view(np.uint8)) for q in a), (state, form, k)


def test_binding_refuses(S):
    x = torch.zeros(64, device="cuda")
    b = torch.zeros(64, dtype=torch.uint8, device="cuda")
    s = torch.zeros(2, dtype=torch.uint8, device="cuda")
    new = lambda: torch.zeros(64, device="cuda")  # noqa: E731
    for f in (lambda: S.adamw_tensor(x, x[:5], new(), new()), lambda: S.adamw_tensor(x, new(), new(), new(), m_scale=s),
              lambda: S.adamw_tensor(x, new(), b, b.clone()), lambda: S.adamw_tensor(x, new(), b, b.clone(), s, s[:1]),
              lambda: S.adamw_tensor(x, new(), new().half(), new().half()),
              lambda: S.adamw_tensor(x, S.operand(new()), new(), new()),
              lambda: S.adamw_tensor(x, new(), new(), new(), model=new())):
        with pytest.raises(ValueError):
            f()
    table = torch.empty(1 << 12, dtype=torch.uint8, device="cuda")
    mixed = [S.adamw_tensor(new(), new(), new(), new()), S.adamw_tensor(new().bfloat16(), new(), new(), new())]
    with pytest.raises(ValueError):
        S.spccl_adamw_plan(mixed, table)
    m = new()
    with pytest.raises(S.SpcclError):                           # m and v the same array
        S.spccl_adamw_plan([S.adamw_tensor(new(), new(), m, m)], table)
    plan = S.spccl_adamw_plan([S.adamw_tensor(new(), new(), new(), new())], table)
    with pytest.raises(ValueError):
        S.spccl_adamw_step(plan, table[:256], 1e-3, grad_scale=torch.zeros(2, device="cuda"))


def test_a_table_that_is_no_device_memory_is_refused(S):
    """Addresses that the device cannot reach are an error of the call, before
    its first launch: one that nothing lies at, and host memory."""
    log("adamw table elsewhere")
    new = lambda: torch.zeros(1000, device="cuda")  # noqa: E731
    tensors = [S.adamw_tensor(new(), new(), new(), new())]
    arr = (S.spccl_adamw_tensor_t * 1)(*tensors)
    need = S.spccl_adamw_plan_bytes(tensors)
    host = torch.zeros(need + 16, dtype=torch.uint8)
    p = S.spccl_adamw_plan_t()
    call = lambda table: S._lib.spccl_adamw_plan(arr, 1, S.SPCCL_F32, S.SPCCL_F32, S.SPCCL_STATE_F32, table, need,  # noqa: E731
                                                 ctypes.byref(p), None)
    for table in (100 << 20, -(-host.data_ptr() // 16) * 16):
        assert call(table) == 6
        assert p.magic == 0
    # the refusal leaves no error behind, and a real table is taken
    torch.cuda.synchronize()
    table = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert call(table.data_ptr()) == 0
    torch.cuda.synchronize()


def test_a_shared_gradient(S):
    """Two tensors may read one gradient: each takes the step it takes alone."""
    log("adamw shared gradient")
    g = torch.full((1000,), 0.25, device="cuda")
    sets = [[torch.full((1000,), float(k), device="cuda"), *(torch.zeros(1000, device="cuda") for _ in range(2))]
            for k in (1, 2, 1, 2)]
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    for group in (sets[:2], sets[2:3], sets[3:]):
        tensors = [S.adamw_tensor(p, g, m, v) for p, m, v in group]
        table = torch.empty(S.spccl_adamw_plan_bytes(tensors), dtype=torch.uint8, device="cuda")
        S.spccl_adamw_step(S.spccl_adamw_plan(tensors, table), ws, 1e-3)
    torch.cuda.synchronize()
    for a, b in zip(sets[0] + sets[1], sets[2] + sets[3]):
        assert torch.equal(a, b)
    assert float(sets[0][0][0]) < 1.0


def test_a_second_moment_follows_its_decay_with_the_default_seed(S):
    """A caller who gives no seed but counts the steps: a second moment without
    gradients falls as beta2^t.  A step's rounding is unbiased and off by at
    most one spacing q <= v / 8, a deviation of at most v / 16; over T steps of
    N elements the mean's is at most v sqrt(T) / 16 / sqrt(N).  6 of them, the
    random bits' resolution (2^-20 q a step) and the products' own roundings
    (2 u a step) are allowed."""
    log("adamw default seed")
    n, steps, b2 = 1 << 16, 1000, 0.999
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    state = S.alloc_adamw_state(n, S.SPCCL_STATE_F8)
    state["v"].view(torch.uint8).fill_(0x70)                    # 2^7, the lowest a block's largest may be
    state["v_scale"].view(torch.uint8).fill_(122)               # 2^-5: v = 4
    tensors = [S.adamw_tensor(p, g, **state)]
    plan = S.spccl_adamw_plan(tensors, torch.empty(S.spccl_adamw_plan_bytes(tensors), dtype=torch.uint8, device="cuda"))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    for t in range(1, steps + 1):
        S.spccl_adamw_step(plan, ws, 1e-3, 0.9, b2, step=t)
    torch.cuda.synchronize()
    v = decode(state["v"].view(torch.uint8).cpu().numpy(), state["v_scale"].view(torch.uint8).cpu().numpy())
    exact = 4.0 * float(f32(b2)) ** steps
    tol = exact * (6 * np.sqrt(steps) / 16 / np.sqrt(n) + steps * (2.0 ** -23 + 2 * U))
    assert abs(v.astype(np.float64).mean() - exact) <= tol


def test_the_default_seed_is_the_step(S):
    """No seed: the step's number.  A seed that is given is taken as it is, 0 too."""
    log("adamw seed given")
    got = []
    for kw in (dict(step=5), dict(step=5, seed=5), dict(step=5, seed=0), dict(step=5, seed=None)):
        c = Case(S, [4096], "bf16", "f32", 8, "array", 3)
        S.spccl_adamw_step(c.plan, c.ws, 1e-3, **kw)
        torch.cuda.synchronize()
        got.append(c.read()[0])
    same = lambda a, b: all(np.array_equal(a[k], b[k]) for k in a)  # noqa: E731
    assert same(got[0], got[1]) and same(got[0], got[3]) and not same(got[0], got[2])


@pytest.mark.parametrize("state", [32, 8])
def test_a_scale_or_a_workspace_that_the_step_writes_over(S, state):
    """The step refuses them and changes nothing; their neighbours are taken."""
    log(f"adamw overlaps of the step {state}")
    c = Case(S, [1000, 0, 200], "f32", "f32", state, "array", 3, copy=True)
    before = c.read()
    lr, b1, b2, eps, t = HYPER
    step = lambda **kw: S.spccl_adamw_step(c.plan, kw.pop("ws", c.ws), lr, b1, b2, eps, t, 1, **kw)  # noqa: E731
    inside = [v[i].view(torch.uint8) for v in c.views.values() for i in (0, 2)]
    for b in inside:
        for at in (0, (b.numel() - 4) // 4 * 4):
            if (b.data_ptr() + at) % 4 == 0 and at + 4 <= b.numel():
                with pytest.raises(ValueError, match="grad_scale"):
                    step(grad_scale=b[at:at + 4].view(torch.float32))
    p = c.buffers["param"].view(torch.uint8)
    for at in (0, 3776, 3840):                                   # the first 1000 elements end at 4000
        with pytest.raises(ValueError, match="workspace"):
            step(ws=p[at:at + 256])
    table = c.plan._tensors[1]
    for at in (0, table.numel() // 16 * 16 - 256):
        with pytest.raises(S.SpcclError):
            step(ws=table[at:at + 256])
    torch.cuda.synchronize()
    for b, a in zip(before, c.read()):
        assert all(np.array_equal(b[k].view(np.uint8), a[k].view(np.uint8)) for k in b)
    # a scale right behind a tensor
    c.untouched = {k: t.clone() for k, t in c.buffers.items()}
    c.buffers["param"][1000] = c.untouched["param"][1000] = 0.37
    step(grad_scale=c.buffers["param"][1000:1001])
    torch.cuda.synchronize()
    c.check(c.read(), c.expect(before, HYPER, 1, f32(0.37)))


@pytest.mark.parametrize("which", ["m", "v"])
def test_a_block_of_scale_255_is_nan_whatever_its_values(S, which):
    """8-bit moments that another program wrote: a scale of 255 stands for NaN, so
    its block's parameters become NaN and its scale stays; no other block changes."""
    log(f"adamw scale 255 {which}")
    c, clean = (Case(S, [1000], "f32", "f32", 8, "array", 12) for _ in range(2))
    codes, scales = c.views[which][0], c.views[which + "_scale"][0]
    codes[64:96] = torch.arange(32, dtype=torch.uint8, device="cuda") * 4     # 0 and ordinary values
    scales[2] = 255
    for x in (c, clean):
        x.step(HYPER, 3)
    got, ref = c.read()[0], clean.read()[0]
    assert np.isnan(got["param"][64:96]).all()
    assert got[which + "_scale"][2] == 255 and (got[which + "_scale"] == 255).sum() == 1
    assert np.isnan(decode(got[which], got[which + "_scale"])[64:96]).all()
    for k in got:
        per = 32 if k.endswith("_scale") else 1
        other = np.ones(got[k].size, bool)
        other[64 // per:96 // per] = False
        assert np.array_equal(got[k][other], ref[k][other]), k
