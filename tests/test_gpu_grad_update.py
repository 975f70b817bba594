"""The gradients' norm, the clip and the AdamW step over lists of tensors against their definitions in 64 bits.

Bounds: the sum of squares is formed in fp64, so it is off by n 2^-53 of itself at most.  A clipped gradient is the product of two fp32 numbers, one of them rounded (E),
then rounded to its type.  Moments are made of three roundings of terms as large as their absolute values; the weight by a root, two quotients and their
products, 12 roundings of the update, and one of the result."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import step_oracle as st
from tests.gpu_util import rnd, to_dev, to_np
from tests.score_util import DT, U
from tests.step_util import E, TINY, close

pytestmark = pytest.mark.gpu
# sizes of the tensors of a list: none, empty ones, single elements, odd ones, more than one launch takes, several chunks
LISTS = {"none": [], "empty": [0, 0], "one": [1], "odd": [5, 0, 1, 33, 7, 1000, 4095, 3], "many": [1 + 37 * i % 101 for i in range(131)], "large": [40001, 9, 70000],
         "chunks": [2048, 8192, 16384, 16385, 65536, 65543], "huge": [3 << 21, 1 << 20]}


class List:
    """Tensors that lie one behind the other in a common buffer, each `gap` elements behind the one before it"""

    def __init__(self, sizes, values, dtype, gap=0, first=0):
        import torch
        self.sizes, self.n = sizes, len(sizes)
        self.buf = torch.full((sum(sizes) + gap * len(sizes) + first + 16,), float("nan"), dtype=torch.float32 if dtype == "fp32" else torch.bfloat16, device="cuda:0")
        self.t, at = [], first
        for s, v in zip(sizes, values):
            self.t.append(self.buf[at:at + s])
            self.t[-1].copy_(to_dev(v, dtype))
            at += s + gap
        self.outside = self.buf.isnan()

    @property
    def ptrs(self):
        return (C.c_void_p * max(1, self.n))(*[t.data_ptr() if len(t) else None for t in self.t])

    @property
    def c_sizes(self):
        return (C.c_int64 * max(1, self.n))(*self.sizes)

    def np(self):
        return [to_np(t) for t in self.t]

    def check_outside(self):
        import torch
        assert torch.equal(self.buf.isnan(), self.outside)


def values(sizes, seed, std=1.0, dtype="fp32"):
    rng = np.random.default_rng(seed)
    return [rnd(rng.normal(0, std, s), dtype) for s in sizes]


def sumsq(dtype, l, add=0, start=float("nan"), stream=None):
    import torch
    from paper_2507_00217_amd import stage as S
    total = torch.full((1,), start, dtype=torch.float64, device="cuda:0")
    scratch = torch.full((S.lib().stage_kernel_grad_sumsq_scratch_bytes(),), 255, dtype=torch.uint8, device="cuda:0")
    assert S.lib().stage_kernel_grad_sumsq(DT[dtype], l.n, l.c_sizes, l.ptrs, add, total.data_ptr(), scratch.data_ptr(), scratch.numel(), stream) == 0
    torch.cuda.synchronize()
    return total


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("gap,first", [(0, 0), (1, 3), (8, 0)])
def test_sum_of_squares(dtype, name, gap, first):
    sizes = LISTS[name]
    v = values(sizes, 1, dtype=dtype)
    l = List(sizes, v, dtype, gap, first)
    want = sum(float((t.astype(np.float64) ** 2).sum()) for t in v)
    bound = (sum(sizes) + 1) * 2.0 ** -53 * want
    got = sumsq(dtype, l)
    close("sumsq", to64(got), want, 2 * bound)
    close("added", to64(sumsq(dtype, l, 1, 3.5)), want + 3.5, 2 * bound + 1e-15 * (want + 3.5))
    assert float(sumsq(dtype, l)) == float(got)


def to64(t):
    return t.cpu().numpy()


@pytest.mark.parametrize("value", [1e-30, 1e30, 3e38])
def test_squares_that_fp32_does_not_hold(value):
    l = List([1000, 3], [np.full(1000, value, np.float32), np.zeros(3, np.float32)], "fp32")
    want = 1000 * float(np.float32(value)) ** 2
    close("sumsq", to64(sumsq("fp32", l)), want, 1e-12 * want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("gap,first,shift", [(0, 0, 0), (1, 3, 0), (0, 1, 5), (8, 0, 0)])
@pytest.mark.parametrize("most", [0.5, 1e6])
def test_clip(dtype, name, gap, first, shift, most):
    """Into other tensors, equally far behind a 16-byte boundary or (shift) not, and in place."""
    import torch
    from paper_2507_00217_amd import stage as S
    sizes = LISTS[name]
    v = values(sizes, 2, dtype=dtype)
    l, out = List(sizes, v, dtype, gap, first), List(sizes, [np.zeros(s, np.float32) for s in sizes], dtype, gap, first + shift)
    total = sum(float((t.astype(np.float64) ** 2).sum()) for t in v)
    sq, norm = torch.tensor([total], dtype=torch.float64, device="cuda:0"), torch.full((1,), float("nan"), device="cuda:0")
    clip = lambda o, nrm: S.lib().stage_kernel_grad_clip(DT[dtype], l.n, l.c_sizes, l.ptrs, o.ptrs, sq.data_ptr(), most, nrm, None)
    assert clip(out, norm.data_ptr()) == 0
    torch.cuda.synchronize()
    f = st.clip_factor(total, float(np.float32(most)))
    close("norm", to_np(norm), math.sqrt(total), E * math.sqrt(total))
    for got, t in zip(out.np(), v):
        want = f * t.astype(np.float64)
        close("out", got, want, np.abs(want) * (2 * E + U[dtype] * (1 + 2 * E)) + TINY)
        if f == 1.0:
            assert (got == t).all()
    out.check_outside()
    assert clip(l, None) == 0
    torch.cuda.synchronize()
    for a, b in zip(l.t, out.t):
        assert torch.equal(a, b)
    l.check_outside()


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_what_is_not_finite_stays(value):
    import torch
    from paper_2507_00217_amd import stage as S
    v = values([300, 20], 3)
    v[1][7] = value
    l = List([300, 20], v, "fp32")
    sq, norm = sumsq("fp32", l), torch.zeros(1, device="cuda:0")
    assert not math.isfinite(float(sq))
    assert S.lib().stage_kernel_grad_clip(0, l.n, l.c_sizes, l.ptrs, l.ptrs, sq.data_ptr(), 1.0, norm.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert not math.isfinite(float(norm))
    for a, b in zip(l.np(), v):
        assert np.array_equal(a, b, equal_nan=True)
    u = Update([300, 20], "bf16", "fp32", 0, 0, grads=v)
    before = {k: [t.clone() for t in x.t] for k, x in u.lists.items()}
    assert u.step(sumsq=sq, max_norm=1.0) == 0
    torch.cuda.synchronize()
    for k, x in u.lists.items():
        for a, b in zip(x.t, before[k]):
            assert torch.equal(a.view(torch.int16 if a.element_size() == 2 else torch.int32), b.view(torch.int16 if a.element_size() == 2 else torch.int32)), k


class Update:
    HYPER = dict(lr=0.03, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)

    def __init__(self, sizes, dtype, gdtype, gap, first, grads=None, shift=0):
        self.dtype, self.gdtype, self.sizes = dtype, gdtype, sizes
        self.v0 = dict(x=values(sizes, 11, 0.5), m=values(sizes, 12, 0.1), v=[t ** 2 for t in values(sizes, 13, 0.1)], g=grads or values(sizes, 14, 0.3, gdtype))
        self.lists = dict(x=List(sizes, self.v0["x"], "fp32", gap, first), m=List(sizes, self.v0["m"], "fp32", gap, first), v=List(sizes, self.v0["v"], "fp32", gap, first + shift),
                          g=List(sizes, self.v0["g"], gdtype, gap, first))
        if dtype == "bf16":
            self.lists["w"] = List(sizes, [np.zeros(s, np.float32) for s in sizes], dtype, gap, first)

    def step(self, step=3, sumsq=None, max_norm=0.0, lr_now=None, step_now=None, stream=None, **hyper):
        from paper_2507_00217_amd import stage as S
        l, p = self.lists, lambda t: None if t is None else t.data_ptr()
        self.hyper = dict(self.HYPER, **hyper)
        self.args = S.AdamW(dtype=DT[self.dtype], grad_dtype=DT[self.gdtype], step=step, sumsq=p(sumsq), max_norm=max_norm, lr_now=p(lr_now), step_now=p(step_now), **self.hyper)
        lp = self.dtype == "bf16"
        return S.lib().stage_kernel_adamw(C.byref(self.args), l["x"].n, l["x"].c_sizes, (l["w"] if lp else l["x"]).ptrs, l["x"].ptrs if lp else None, l["m"].ptrs, l["v"].ptrs,
                                          l["g"].ptrs, stream)

    def check(self, step=3, factor=1.0, **over):
        h = dict(self.hyper, **over)
        got = {k: x.np() for k, x in self.lists.items()}
        for i in range(len(self.sizes)):
            x, m, v, g = (self.v0[k][i].astype(np.float64) for k in ("x", "m", "v", "g"))
            g = g * factor
            wx, wm, wv = st.adamw(x, m, v, g, step=step, **h)
            close("m", got["m"][i], wm, 4 * E * (np.abs(h["beta1"] * m) + np.abs((1 - h["beta1"]) * g)) + TINY)
            e_v = 6 * E * (h["beta2"] * v + (1 - h["beta2"]) * g * g) + TINY
            close("v", got["v"][i], wv, e_v)
            den = np.sqrt(wv / (1 - h["beta2"] ** step)) + h["eps"]
            # the update's relative error, and that of the moment in its numerator where its two terms nearly cancel
            up = (np.abs(h["beta1"] * m) + np.abs((1 - h["beta1"]) * g)) / (1 - h["beta1"] ** step) / den
            bound = h["lr"] * (12 * E * up + 4 * E * h["weight_decay"] * np.abs(x)) + 2 * E * np.abs(wx)
            close("weight", got["x"][i], wx, bound)
            if self.dtype == "bf16":
                assert (got["w"][i] == rnd(got["x"][i], "bf16")).all()
        for l in self.lists.values():
            l.check_outside()


@pytest.mark.parametrize("dtype,gdtype", [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")])
@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("gap,first,shift", [(0, 0, 0), (1, 3, 0), (0, 1, 2), (8, 0, 0)])
def test_adamw(dtype, gdtype, name, gap, first, shift):
    import torch
    u = Update(LISTS[name], dtype, gdtype, gap, first, shift=shift)
    assert u.step(step=1 + len(name)) == 0
    torch.cuda.synchronize()
    u.check(step=1 + len(name))


@pytest.mark.parametrize("hyper", [dict(beta1=0.0, beta2=0.0), dict(lr=0.0), dict(weight_decay=0.0), dict(eps=0.1), dict(beta1=0.999, beta2=0.99999)])
@pytest.mark.parametrize("step", [1, 2, 100000])
def test_adamw_hyperparameters(hyper, step):
    import torch
    u = Update([999, 4], "bf16", "fp32", 0, 0)
    assert u.step(step=step, **hyper) == 0
    torch.cuda.synchronize()
    u.check(step=step)


@pytest.mark.parametrize("most", [0.25, 1e9])
def test_adamw_of_clipped_gradients(most):
    """The norm's call, then the step that reads it: what clip and step give."""
    import torch
    u = Update([5000, 31], "bf16", "bf16", 1, 1)
    sq = sumsq("bf16", u.lists["g"])
    assert u.step(sumsq=sq, max_norm=most) == 0
    torch.cuda.synchronize()
    u.check(factor=st.clip_factor(float(sq), most))


def test_learning_rate_and_step_on_the_device():
    import torch
    u = Update([700], "fp32", "fp32", 0, 0)
    lr, step = torch.tensor([0.007], device="cuda:0"), torch.tensor([41], dtype=torch.int32, device="cuda:0")
    assert u.step(step=1, lr_now=lr, step_now=step) == 0
    torch.cuda.synchronize()
    u.check(step=41, lr=float(np.float32(0.007)))
    u = Update([700], "fp32", "fp32", 0, 0)
    step.fill_(-3)
    assert u.step(step=9, step_now=step) == 0
    torch.cuda.synchronize()
    u.check(step=1)
