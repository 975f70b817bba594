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
