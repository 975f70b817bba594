"""Attention of shaped scores over packed sequences (cap, distance bias, prefix) against its definition in 64 bits, forward and
backward, with elementwise bounds from the roundings (tests/score_util.py)."""
import numpy as np
import pytest

from paper_2507_00217_amd import synth
from tests.gpu_util import rnd
from tests.score_util import Attention

pytestmark = pytest.mark.gpu


def inputs(dtype, rows, h, hkv, hd, seed, spread=1.0):
    mk = lambda i, n, std: rnd(synth.normal(seed, i, (rows, n * hd), std=std), dtype)
    return mk(1, h, spread), mk(2, hkv, spread), mk(3, hkv, 1.0), mk(4, h, 1.0)


def slopes(h):
    return (2.0 ** (-8.0 * np.arange(1, h + 1) / h)).astype(np.float32)


# lengths of the packed sequences, rows before the first and behind the last
PACKED = {"one": ([1], 0, 0), "ones": ([1, 1, 1, 1, 1], 0, 2), "empty": ([0, 5, 0, 0, 70, 0], 3, 0), "tiles": ([64, 128, 32, 256], 0, 0),
          "odd": ([63, 65, 129, 1, 31, 33], 2, 5), "long": ([3, 610], 0, 1)}
# 0: by the shape, 1: the plain kernels; the others fix the workgroup shapes, 2 .. 5 of forward, dQ and dK/dV, 6 and 7 of the one-launch backward
KERNELS = [("fp32", 0), ("fp32", 1)] + [("bf16", n) for n in range(8)]


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("shape", list(PACKED))
@pytest.mark.parametrize("causal,prefix", [(1, 0), (0, 0), (1, 1)])
def test_packed_sequences(dtype, kernel_set, hd, shape, causal, prefix):
    lens, before, behind = PACKED[shape]
    rows, h, hkv = sum(lens) + before + behind, 4, 2
    starts = before + np.concatenate(([0], np.cumsum(lens)))
    q, k, v, do = inputs(dtype, rows, h, hkv, hd, 31)
    out = np.ones(rows, bool)
    out[starts[0]:starts[-1]] = False
    for a in (q, k, v, do):
        a[out] = np.nan                                            # rows of no sequence are not read
    prefixes = [(n * 2) // 3 if i % 2 else n + 7 * (i % 3) - 3 for i, n in enumerate(lens)] if prefix else None
    Attention(dtype, q, k, v, do, h, hkv, causal, starts=starts, prefixes=prefixes, n_seq=len(lens)).check(kernel_set)


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("cap,bias,spread", [(0.0, 0, 1.0), (30.0, 0, 1.5), (5.0, 0, 2.5), (0.0, 1, 1.0), (20.0, 1, 2.0)])
@pytest.mark.parametrize("n_seq,s,h,hkv", [(1, 200, 4, 1), (3, 77, 6, 6)])
def test_cap_and_bias(dtype, kernel_set, hd, causal, cap, bias, spread, n_seq, s, h, hkv):
    """cap 5 with scores of up to 30 is far into the flat part of the tanh."""
    q, k, v, do = inputs(dtype, n_seq * s, h, hkv, hd, 37, spread)
    Attention(dtype, q, k, v, do, h, hkv, causal, cap=cap, slopes=slopes(h) if bias else None, n_seq=n_seq).check(kernel_set)


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("pads", [(8, 16, 24, 32, 40), (1, 3, 5, 7, 9)])
def test_strides_and_every_option(dtype, kernel_set, pads):
    """Columns of wider buffers (odd strides: the plain kernels), a scale of its own, all options at once."""
    lens, h, hkv, hd = [100, 0, 37, 130], 6, 2, 128
    starts = np.concatenate(([0], np.cumsum(lens))) + 1
    q, k, v, do = inputs(dtype, sum(lens) + 4, h, hkv, hd, 41)
    Attention(dtype, q, k, v, do, h, hkv, 1, scale=0.11, cap=15.0, slopes=slopes(h), starts=starts, prefixes=[30, 5, 37, 0], n_seq=4, pads=pads).check(kernel_set)
