"""Attention of shaped scores against 64 bits from the inputs alone (tests/score_exact.py), at sizes and values where kernels differ in what they
round."""
import numpy as np
import pytest

from tests.gpu_util import rnd
from tests.score_exact import compare
from tests.score_util import Attention
from tests.test_gpu_score_attention import KERNELS, inputs, slopes

pytestmark = pytest.mark.gpu

# few rows among long ones: the mean is above 128 rows, so nothing but the offsets tells that some sequences are short
MIXED = [[8, 700, 20, 12, 600, 33, 60, 480, 5, 120], [40, 9, 900, 3, 64, 128]]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens", MIXED)
@pytest.mark.parametrize("h,hkv,cap,causal", [(4, 4, 0.0, 1), (4, 2, 20.0, 1), (8, 8, 0.0, 0)])
def test_short_sequences_packed_with_long_ones(hd, lens, h, hkv, cap, causal):
    """Gradients of a short sequence do not lose what the rounding of O loses, whatever it is packed with."""
    import torch
    starts = np.concatenate(([0], np.cumsum(lens)))
    q, k, v, do = inputs("bf16", int(starts[-1]), h, hkv, hd, 113, 2.0)
    p = Attention("bf16", q, k, v, do, h, hkv, causal, cap=cap, starts=starts, n_seq=len(lens))
    assert p.fwd() == 0 and p.bwd() == 0
    torch.cuda.synchronize()
    compare(p, only=lambda n: n <= 128)


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("hd,cap", [(64, 0.0), (128, 0.0), (128, 20.0)])
@pytest.mark.parametrize("causal,prefix", [(1, 0), (1, 90), (0, 0)])
def test_steep_slopes(dtype, kernel_set, hd, cap, causal, prefix):
    """The bias of a pair of rows at distance 0 is 0 and that of neighbours one slope, however steep it is: nothing of the distances to a block's first row
    is left in them.  (A pair whose bias is beyond 100 has no weight.)"""
    import torch
    rows, s = 300, [3.0, 50.0, 1e4, 3e6]
    q, k, v, do = inputs(dtype, rows, 4, 2, hd, 127)
    p = Attention(dtype, q, k, v, do, 4, 2, causal, cap=cap, slopes=s, prefixes=[prefix] if prefix else None)
    assert p.fwd(kernel_set) == 0 and p.bwd(kernel_set) == 0
    torch.cuda.synchronize()
    compare(p, exact_delta=(False, False))


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("hd,cap", [(64, 0.0), (128, 0.0), (128, 2.0 ** 110)])
@pytest.mark.parametrize("size", [2.0 ** 40, 2.0 ** 53, 2.0 ** 59])
def test_scores_far_below_zero(dtype, kernel_set, hd, cap, size):
    """Scores of -1e23 to -1e35 are scores like any others: a row's weight is on its highest, wherever that lies.  (The products are exact; of the softmax
    nothing but the largest is left, so o is that key's value.)"""
    import torch
    rows = 200
    _, _, v, do = inputs(dtype, rows, 1, 1, hd, 131)
    q, k = np.zeros((rows, hd), np.float32), np.zeros((rows, hd), np.float32)
    rank = np.random.default_rng(3).permutation(256)[:rows] // 2                   # 7 bits: exact in bf16, two keys at most share one
    q[:, 3], k[:, 3] = size, -size * (1.0 + rank / 128.0)
    p = Attention(dtype, q, k, v, do, 1, 1, 1, cap=cap)
    assert p.fwd(kernel_set) == 0
    torch.cuda.synchronize()
    compare(p, names=("o", "lse"))


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("cap", [2e3, 1e5, 1e7])
def test_large_cap_beside_outliers(dtype, kernel_set, hd, cap):
    """A cap far above the scores of most rows, with some rows that reach it: the others keep their precision, though they share blocks with them.  (The
    outliers' own scores are beyond what F32 is for; their dO is zero, so they add nothing to dk and dv.)"""
    import torch
    rows = 230
    q, k, v, do = inputs(dtype, rows, 2, 1, hd, 137)
    big = np.arange(rows) % 7 == 3
    q[big] = rnd(q[big] * cap, dtype)
    do[big] = 0.0
    p = Attention(dtype, q, k, v, do, 2, 1, 1, cap=cap)
    assert p.fwd(kernel_set) == 0 and p.bwd(kernel_set) == 0
    torch.cuda.synchronize()
    compare(p, exact_delta=(False, False), rows=~big)
    compare(p, names=("lse",))                       # of the outliers too: a score near a large cap is off by no more of itself than any other


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("scale,cap", [(1e-10, 5.0), (1e-20, 30.0), (1e-3, 300.0)])
def test_small_scale_under_a_cap(dtype, kernel_set, hd, scale, cap):
    """Queries and keys whose products are as large as the scale is small: scores of ordinary size, some of them near the cap.

    Scores go up to two thirds of 300, past the 100 that F32 is for, so what fp32 may do to a P is counted: its exponent is made by at most 8 roundings
    (scale, cap, sums, lse) of numbers up to 2 cap + log(rows), its product q.k by at most 64 of partial sums up to D = scale sum |q k|, each 2^-24."""
    import torch
    rows = 230
    q, k, v, do = inputs(dtype, rows, 2, 1, hd, 139)
    big = np.float32(2.0 ** round(np.log2(cap / 6.0 / scale / hd ** 0.5) / 2))                # scores of cap / 6 in the mean, up to two thirds of it
    D = scale * float(big) ** 2 * max(float((np.abs(q[:, j * hd:(j + 1) * hd]) @ np.abs(k).T).max()) for j in range(2))
    p = Attention(dtype, q * big, k * big, v, do, 2, 1, 1, scale=scale, cap=cap)
    assert p.fwd(kernel_set) == 0 and p.bwd(kernel_set) == 0
    torch.cuda.synchronize()
    compare(p, exact_delta=(False, False), f32=2.0 ** -24 * (8 * (2 * cap + np.log(rows)) + 64 * D))


def packed(lens, behind=0):
    return dict(starts=np.concatenate(([0], np.cumsum(lens))), n_seq=len(lens)), int(np.sum(lens)) + behind


# what the rules choose where they choose it: every kernel at sizes it is made for, two KV heads with all of their query heads
SIZES = {
    "wide, capped": ("bf16", 4096, 32, 8, 128, 3.0, dict(cap=50.0)),
    "long, biased": ("bf16", 16384, 8, 2, 128, 1.0, dict(slopes=slopes(8))),
    "documents": ("bf16", [700, 50, 1259, 90, 1100, 400, 33, 1000, 820, 610, 750, 128, 1156], 16, 2, 128, 1.0, dict(behind=96)),
    "prefixes": ("bf16", [900, 100, 1300, 64, 700, 500, 532], 40, 40, 128, 1.0, dict(prefixes=[300, 60, 800, 10, 0, 490, 100])),
    "narrow heads in one launch": ("bf16", 2331, 12, 12, 64, 1.0, dict(n_seq=3, slopes=slopes(12))),
    "narrow heads": ("bf16", 8192, 12, 4, 64, 1.0, {}),
    "many short": ("bf16", [20 + 7 * (i % 23) for i in range(100)], 16, 16, 64, 2.0, dict(cap=30.0)),
    "full": ("bf16", 4096, 16, 16, 128, 1.0, dict(n_seq=2, causal=0)),
    "few heads": ("bf16", 5000, 4, 4, 128, 1.0, {}),
    "fp32": ("fp32", 1500, 16, 4, 128, 2.0, dict(cap=30.0, slopes=slopes(16), prefixes=[200])),
}


@pytest.mark.parametrize("name", list(SIZES))
def test_at_the_sizes_of_the_rules(name):
    import torch
    dtype, rows, h, hkv, hd, spread, opts = SIZES[name]
    opts = dict(opts)
    if not isinstance(rows, int):
        more, rows = packed(rows, opts.pop("behind", 0))
        opts.update(more)
    q, k, v, do = inputs(dtype, rows, h, hkv, hd, 157, spread ** 0.5)
    p = Attention(dtype, q, k, v, do, h, hkv, opts.pop("causal", 1), **opts)
    assert p.fwd() == 0 and p.bwd() == 0
    torch.cuda.synchronize()
    compare(p, groups=sorted({0, hkv - 1}), exact_delta=(True, "starts" in opts))
