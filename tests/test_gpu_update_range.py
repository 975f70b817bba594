"""Clip and AdamW at the ends of fp32's range, and long lists in the form that streams, against their definitions in 64 bits."""
import math

import numpy as np
import pytest

from oracle import step_oracle as st
from tests.gpu_util import to_np
from tests.score_util import DT, U
from tests.step_util import E, TINY, close
from tests.test_gpu_grad_update import List, Update, sumsq, to64, values

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# norms whose factor fp32 does not hold
# ---------------------------------------------------------------------------
def diverged(sizes, largest, dtype):
    """Gradients of up to `largest`, spread over forty powers of ten, zeros among them"""
    from tests.gpu_util import rnd
    rng = np.random.default_rng(21)
    out = [rng.normal(0, 1, s) * 10.0 ** rng.uniform(-40, 0, s) for s in sizes]
    out[0][::7] = 0.0
    out[0][1::7] = 1.0
    return [rnd(np.clip(t, -1, 1) * largest, dtype) for t in out]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("largest,most", [(3e38, 1.0), (1e38, 0.5), (3e38, 1e-3), (1e30, 1.0), (1e31, 1e-3), (1e38, 1e30)])
def test_clip_of_diverged_gradients(dtype, largest, most):
    """The factor is max_norm / norm, down to 1e-43 here, where fp32 has a few bits left: the product is as exact as any, of gradients of every size."""
    import torch
    from paper_2507_00217_amd import stage as S
    sizes = [20000, 3, 1000]
    v = diverged(sizes, largest, dtype)
    l, out = List(sizes, v, dtype), List(sizes, [np.zeros(s, np.float32) for s in sizes], dtype, 1, 1)
    sq = sumsq(dtype, l)
    total = sum(float((t.astype(np.float64) ** 2).sum()) for t in v)
    close("sumsq", to64(sq), total, 1e-11 * total)
    for o in (out, l):
        assert S.lib().stage_kernel_grad_clip(DT[dtype], l.n, l.c_sizes, l.ptrs, o.ptrs, sq.data_ptr(), most, None, None) == 0
        torch.cuda.synchronize()
        f = st.clip_factor(total, float(np.float32(most)))
        for got, t in zip(o.np(), v):
            want = f * t.astype(np.float64)
            close("out", got, want, np.abs(want) * (3 * E + U[dtype] * (1 + 3 * E)) + TINY)
        o.check_outside()


@pytest.mark.parametrize("largest,most", [(3e38, 1.0), (1e31, 1e-3)])
@pytest.mark.parametrize("dtype,gdtype", [("fp32", "fp32"), ("bf16", "bf16")])
def test_adamw_of_diverged_gradients(dtype, gdtype, largest, most):
    import torch
    sizes = [20000, 3, 1000]
    u = Update(sizes, dtype, gdtype, 1, 1, grads=diverged(sizes, largest, gdtype))
    sq = sumsq(gdtype, u.lists["g"])
    assert u.step(sumsq=sq, max_norm=most) == 0
    torch.cuda.synchronize()
    u.check(factor=st.clip_factor(float(sq), float(np.float32(most))))


# ---------------------------------------------------------------------------
# lists of more than the last-level cache holds, whose accesses ask to keep nothing
# ---------------------------------------------------------------------------
def long_list(sizes, first, dtype, seed, std=1.0):
    """A buffer of normal numbers and its tensors, one behind the other from element `first` on"""
    import torch
    buf = torch.empty(first + sum(sizes) + 8, dtype=torch.float32 if dtype == "fp32" else torch.bfloat16, device="cuda:0")
    buf.normal_(generator=torch.Generator(device="cuda:0").manual_seed(seed)).mul_(std)
    at = [first + sum(sizes[:i]) for i in range(len(sizes))]
    return buf, [buf[a:a + n] for a, n in zip(at, sizes)]


def arrays(sizes, *lists):
    import ctypes as C
    n = len(sizes)
    return (C.c_int64 * n)(*sizes), [None if l is None else (C.c_void_p * n)(*[t.data_ptr() for t in l]) for l in lists]


def around_is_kept(before, after, first, n):
    import torch
    return torch.equal(before[:first], after[:first]) and torch.equal(before[first + n:], after[first + n:])


@pytest.mark.parametrize("first,shift", [(0, 0), (3, 0), (1, 1)])
def test_norm_and_clip_of_long_lists(first, shift):
    """280 MB of fp32 gradients, equally far behind a boundary as where they go, or not."""
    import torch
    from paper_2507_00217_amd import stage as S
    from tests.gpu_util import launches
    L, sizes, E64 = S.lib(), [40000001, 5, 30000002], 2.0 ** -53
    n = sum(sizes)
    buf, g = long_list(sizes, first, "fp32", 31)
    obuf, o = long_list(sizes, first + shift, "fp32", 32)
    c_sizes, (gp, op) = arrays(sizes, g, o)
    total, scratch = torch.full((1,), math.nan, dtype=torch.float64, device="cuda:0"), torch.empty(L.stage_kernel_grad_sumsq_scratch_bytes(), dtype=torch.uint8, device="cuda:0")
    norm, most = torch.zeros(1, device="cuda:0"), 0.75
    norms = lambda s: L.stage_kernel_grad_sumsq(0, len(sizes), c_sizes, gp, 0, total.data_ptr(), scratch.data_ptr(), scratch.numel(), s)
    clip = lambda s: L.stage_kernel_grad_clip(0, len(sizes), c_sizes, gp, op, total.data_ptr(), most, norm.data_ptr(), s)
    assert "sumsq_kernelIfLb1E" in launches(norms)[0][0] and "clip_kernelIfLb1E" in launches(clip)[0][0]
    stream, kept = torch.cuda.current_stream().cuda_stream, obuf.clone()
    assert norms(stream) == 0 and clip(stream) == 0
    torch.cuda.synchronize()
    want = sum(float((t.double() ** 2).sum()) for t in g)
    assert abs(float(total) - want) <= 2 * n * E64 * want and abs(float(norm) - math.sqrt(want)) <= E * math.sqrt(want)
    f = st.clip_factor(float(total), most)
    for a, b in zip(g, o):
        w = a.double() * f
        assert bool(((b.double() - w).abs() <= w.abs() * 3 * E + TINY).all())
    assert around_is_kept(kept, obuf, first + shift, n)


@pytest.mark.parametrize("dtype,gdtype", [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")])
@pytest.mark.parametrize("first,shift", [(0, 0), (3, 0), (1, 1)])
def test_adamw_of_long_lists(dtype, gdtype, first, shift):
    """13 million parameters with their moments, 340 MB and more, all alike behind a boundary or the second moments elsewhere; the same bounds as of short lists."""
    import ctypes as C

    import torch
    from paper_2507_00217_amd import stage as S
    from tests.gpu_util import launches
    sizes = [8000001, 7, 5000000]
    n, lp = sum(sizes), dtype == "bf16"
    hyper, step, most = dict(lr=0.03, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1), 4, 2.0
    bufs = {k: long_list(sizes, first + (shift if k == "v" else 0), d, i, std) for i, (k, d, std) in enumerate((("x", "fp32", 0.5), ("m", "fp32", 0.1), ("v", "fp32", 0.1), ("g", gdtype, 0.3)))}
    bufs["v"][0].square_()
    if lp:
        bufs["w"] = long_list(sizes, first, "bf16", 9)
    before = {k: b.clone() for k, (b, _) in bufs.items()}
    t = {k: l for k, (_, l) in bufs.items()}
    c_sizes, (w, x, m, v, g) = arrays(sizes, t["w"] if lp else t["x"], t["x"] if lp else None, t["m"], t["v"], t["g"])
    total = sum((a.double() ** 2).sum() for a in t["g"]).reshape(1)
    p = S.AdamW(dtype=DT[dtype], grad_dtype=DT[gdtype], step=step, sumsq=total.data_ptr(), max_norm=most, **hyper)
    call = lambda s: S.lib().stage_kernel_adamw(C.byref(p), len(sizes), c_sizes, w, x, m, v, g, s)
    ((name, _, _),) = launches(call)
    assert "adamw_kernelI" + {"fp32": "f", "bf16": "DF16b"}[dtype] in name and "Lb1E" in name, name
    assert call(torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    f, b1, b2 = st.clip_factor(float(total), most), hyper["beta1"], hyper["beta2"]
    for i in range(len(sizes)):
        was = lambda k: before[k].as_strided((sizes[i],), (1,), t[k][i].storage_offset()).double()
        x0, m0, v0, g0 = was("x"), was("m"), was("v"), was("g") * f
        m1, v1 = b1 * m0 + (1 - b1) * g0, b2 * v0 + (1 - b2) * g0 * g0
        den = torch.sqrt(v1 / (1 - b2 ** step)) + hyper["eps"]
        x1 = x0 - hyper["lr"] * (hyper["weight_decay"] * x0 + m1 / (1 - b1 ** step) / den)
        size = b1 * m0.abs() + (1 - b1) * g0.abs()
        assert bool(((t["m"][i].double() - m1).abs() <= 4 * E * size + TINY).all())
        assert bool(((t["v"][i].double() - v1).abs() <= 6 * E * v1 + TINY).all())
        bound = hyper["lr"] * (12 * E * size / (1 - b1 ** step) / den + 4 * E * hyper["weight_decay"] * x0.abs()) + 2 * E * x1.abs()
        assert bool(((t["x"][i].double() - x1).abs() <= bound).all())
        if lp:
            assert torch.equal(t["w"][i], t["x"][i].bfloat16())
    assert torch.equal(before["g"], bufs["g"][0])
    for k, (b, _) in bufs.items():
        assert around_is_kept(before[k], b, first + (shift if k == "v" else 0), n)
