"""Log probabilities and the logits' gradient on rows and sizes where kernels part: rows of nothing but NaN, ties below zero."""
import math

import numpy as np
import pytest

from tests.step_util import Logprob, logits

pytestmark = pytest.mark.gpu
SETS = [0, 1, 2]


def sync():
    import torch
    torch.cuda.synchronize()


def signalling(t, rows):
    """puts NaNs that are not quiet over the rows of a tensor"""
    import torch
    half = t.element_size() == 2
    t.view(torch.int16 if half else torch.int32)[rows] = 0x7f81 if half else 0x7f800001


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 9, 100, 700, 1500, 3500, 7001, 20003])
@pytest.mark.parametrize("top", [0, 3])
def test_rows_of_nan(kernel_set, dtype, vocab, top):
    """Nothing but NaN, NaN among -inf wherever it lies, signalling ones: the largest logit that is a number is -inf, as in a row without tokens, but such a row's gradient is zeros and these
    rows' is NaN, whose norm no update takes."""
    import torch
    from tests.test_gpu_grad_update import List, sumsq
    x, _, _ = logits(9, vocab, dtype, vocab)
    target, top = np.arange(9) % vocab, min(top, vocab)
    x[0] = x[5] = np.nan
    x[1:5] = -np.inf
    x[1, 0] = x[2, vocab // 2] = x[3, vocab - 1] = np.nan            # row 4: no token
    x[6, ::2] = np.nan
    x[6, 1::2] = -np.inf
    x[7, 0] = np.nan
    w, dh, dl = np.full(9, -0.5, np.float32), np.full(9, 0.25, np.float32), np.full(9, 0.125, np.float32)
    for grads in ((w, dh, dl), (w, None, None), (None, None, dl)):
        pr = Logprob(dtype, x, target, 1.0, top, *grads, (3, 3), (1, 1))
        signalling(pr.x, 5)
        assert pr.fwd(kernel_set) == 0 and pr.bwd(kernel_set) == 0
        sync()
        ref = pr.check_values()
        pr.check_grad(ref)
        first = pr.dx.clone()
        pr.dx.fill_(7.0)
        assert pr.grad(kernel_set) == 0
        sync()
        pr.check_values(ref)
        pr.check_grad(ref)
        for g in (first, pr.dx):
            assert bool(g[[0, 1, 2, 3, 5, 6, 7]].isnan().all()) and bool((g[4] == 0).all()) and bool(g[8].isfinite().all())
            one = List([vocab], [np.zeros(vocab)], dtype)
            for r in (0, 1, 3, 5):
                one.t[0].copy_(g[r])
                assert not math.isfinite(float(sumsq(dtype, one)))


def test_a_row_of_nan_in_a_share_of_the_vocabulary():
    """Statistics that a program has joined over shares: the share whose columns are all -inf has NaN where another share's logits made ln S NaN, zeros where no share has a token."""
    import torch
    for kernel_set in (0, 1):
        x = np.full((2, 300), -np.inf, np.float32)
        pr = Logprob("fp32", x, [-1, -1], 1.0, 0, None, None, [0.5, 0.5])
        pr.out["stats"].copy_(torch.tensor([[-math.inf, math.nan], [-math.inf, -math.inf]]))
        assert pr.bwd(kernel_set) == 0
        sync()
        assert bool(pr.dx[0].isnan().all()) and bool((pr.dx[1] == 0).all())


def tied(how, vocab, dtype):
    """One row whose alternatives are decided among equal logits"""
    import torch
    from tests.gpu_util import rnd
    rng, low = np.random.default_rng(3), float(torch.finfo(torch.float32 if dtype == "fp32" else torch.bfloat16).min)
    left = np.isin(np.arange(vocab), rng.integers(0, vocab, 9))
    kinds = {"constant": np.full(vocab, -1.0), "small": np.full(vocab, -1e-30), "two values": np.where(rng.random(vocab) < 0.5, -1.0, -2.0), "lowest": np.full(vocab, low),
             "few left": np.where(left, rng.normal(0, 1, vocab), -1e4), "few left, lowest": np.where(left, rng.normal(0, 1, vocab), low),
             "few left, negative": np.where(left, rng.normal(-9, 1, vocab), -1e4), "above": np.full(vocab, 1.0), "zero": np.zeros(vocab)}
    return rnd(kinds[how], dtype)


TIES = ["constant", "small", "two values", "lowest", "few left", "few left, lowest", "few left, negative"]


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,top", [(700, 40), (3300, 64), (5000, 64), (40000, 20)])
@pytest.mark.parametrize("how", TIES)
def test_ties_below_zero(kernel_set, dtype, vocab, top, how):
    x = tied(how, vocab, dtype)
    pr = Logprob(dtype, np.stack((x, x)), [1, vocab - 1], 1.0, top)
    assert pr.fwd(kernel_set) == 0
    sync()
    pr.check_values()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("how", TIES)
def test_what_ties_take(dtype, how):
    """The way made for ties finds them in one more pass over a row: twice what rows of zeros take is room for another share of rows that take it (or the walk a second time, which the lowest values make).
    One by one, `top` passes, was 8 times and more."""
    import torch
    from tests.test_gpu_score_odd import once
    rows, vocab, top = 512, 40000, 40
    time = {}
    for kind in ("zero", how):
        pr = Logprob(dtype, np.broadcast_to(tied(kind, vocab, dtype), (rows, vocab)), None, 1.0, top)
        stream = torch.cuda.current_stream().cuda_stream
        time[kind] = once(lambda: pr.fwd(0, stream))
    assert time[how] <= 2 * time["zero"], time
