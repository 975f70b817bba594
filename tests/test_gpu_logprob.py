"""Log probabilities of given tokens, entropy, alternatives and the logits' gradient against their definitions in 64 bits."""
import numpy as np
import pytest

from tests.step_util import Logprob, logits

pytestmark = pytest.mark.gpu
SETS = [0, 1, 2]


def sync():
    import torch
    torch.cuda.synchronize()


def untouched(pr):
    """what lies around the gradient's rows is as it was"""
    import torch
    t, n, shift = pr.whole_dx, pr.vocab, pr.dx.storage_offset()
    return bool(torch.isnan(t[:, :shift].float()).all()) and bool(torch.isnan(t[:, shift + n:].float()).all())


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 2), (5, 7, 3), (2, 64, 64), (130, 65, 20), (4, 100, 64), (33, 1000, 5), (7, 1023, 1), (3, 4097, 20), (2, 8200, 64), (2, 33001, 20)])
@pytest.mark.parametrize("pads,shifts,scale", [((0, 0), (0, 0), 0.0), ((3, 8), (1, 1), 1.4), ((0, 5), (3, 6), 0.5)])
def test_values_and_gradient(kernel_set, dtype, rows, vocab, top, pads, shifts, scale):
    """Odd and aligned rows, with logits and gradient equally far behind a 16-byte boundary or not; the two calls and the one call."""
    x, target, (w, dh, dl) = logits(rows, vocab, dtype, vocab + top)
    pr = Logprob(dtype, x, target, scale, top, w, dh, dl, pads, shifts)
    assert pr.fwd(kernel_set) == 0
    sync()
    ref = pr.check_values()
    assert pr.bwd(kernel_set) == 0
    sync()
    pr.check_grad(ref)
    assert untouched(pr)
    pr.dx.fill_(float("nan"))
    for v in pr.out.values():
        v.fill_(-9)
    assert pr.grad(kernel_set) == 0
    sync()
    pr.check_values(ref)
    pr.check_grad(ref)
    assert untouched(pr)


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [90, 2500, 20000])
@pytest.mark.parametrize("kind", ["w", "dh", "dl", "w dh", "w dl"])
def test_each_gradient_by_itself(kernel_set, dtype, vocab, kind):
    x, target, parts = logits(6, vocab, dtype, vocab, banned=0.3)
    x[:, 0] = 1.0
    target[target >= 0] = np.where(np.isfinite(x[np.arange(6), target][target >= 0]), target[target >= 0], 0)
    has = dict(zip(("w", "dh", "dl"), parts))
    pr = Logprob(dtype, x, target if "w" in kind else None, 1.0, 0, **{k: has[k] for k in kind.split()})
    assert pr.fwd(kernel_set) == 0 and pr.bwd(kernel_set) == 0
    sync()
    ref = pr.check_values()
    pr.check_grad(ref)
    pr.dx.fill_(float("nan"))
    assert pr.grad(kernel_set) == 0
    sync()
    pr.check_grad(ref)


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [70, 3000, 9000])
@pytest.mark.parametrize("scale", [1.0, 0.3])
def test_rows_at_the_edge(kernel_set, dtype, vocab, scale):
    """Rows of -inf, of one value, of the type's lowest one, with one token left, with fewer left than alternatives, with infinities and NaN, with zeros of both signs, and
    rows whose weights are zero over anything."""
    import torch
    x, _, _ = logits(16, vocab, dtype, 5)
    low = float(torch.finfo(torch.float32 if dtype == "fp32" else torch.bfloat16).min)
    target = np.arange(16) % vocab
    x[0] = -np.inf
    x[1] = 3.25
    x[2] = low
    x[3] = -np.inf
    x[3, vocab - 3] = 2.0
    target[3] = vocab - 3
    x[4, 5:] = -np.inf
    target[4] = 60                                     # a token that cannot be
    x[5, 17] = np.inf
    x[6, vocab - 1] = np.nan
    x[7] = 0.0
    x[7, ::2] = -0.0
    x[8, :] = low
    x[8, 11] = 1.0
    target[8] = 11
    x[9, vocab // 2] = np.nan
    x[10] = np.inf
    x[11, 3] = 300.0                                    # certain
    target[11] = 3
    target[12] = -1
    target[13] = vocab                                 # none
    w, dh, dl = np.ones(16, np.float32), np.full(16, 0.5, np.float32), np.full(16, -0.25, np.float32)
    for r in (6, 9, 14):
        w[r] = dh[r] = dl[r] = 0.0
    for grads in ((w, dh, dl), (w, None, None)):
        pr = Logprob(dtype, x, target, scale, 20, *grads, (5, 2), (1, 2))
        assert pr.fwd(kernel_set) == 0 and pr.bwd(kernel_set) == 0
        sync()
        ref = pr.check_values()
        pr.check_grad(ref)
        assert bool((pr.dx[[6, 9]] == 0).all())
        pr.dx.fill_(float("nan"))
        assert pr.grad(kernel_set) == 0
        sync()
        pr.check_values(ref)
        pr.check_grad(ref)


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,top", [(3300, 64), (5000, 64), (40000, 20), (40000, 64)])
@pytest.mark.parametrize("how", ["equal", "rising", "falling", "two values", "few left", "one run"])
def test_alternatives_of_odd_rows(kernel_set, dtype, vocab, top, how):
    """Ties everywhere, orders that put the largest side by side, and rows with fewer tokens left than alternatives."""
    rng = np.random.default_rng(1)
    from tests.gpu_util import rnd
    j = np.arange(vocab)
    x = {"equal": np.zeros(vocab), "rising": j / vocab * 8, "falling": -j / vocab * 8, "two values": np.where(rng.random(vocab) < 0.5, 1.0, -1.0),
         "few left": np.where(np.isin(j, rng.integers(0, vocab, 9)), rng.normal(0, 1, vocab), -np.inf),
         "one run": np.where((j > 3000) & (j < 3200), 5 + rng.normal(0, 1, vocab), rng.normal(0, 1, vocab))}[how]
    x = rnd(np.stack((x, x)), dtype)
    pr = Logprob(dtype, x, [1, vocab - 1], 1.0, top)
    assert pr.fwd(kernel_set) == 0
    sync()
    pr.check_values()


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [65, 130, 257, 300, 513, 520, 600, 1000, 1030, 1500, 2100, 4090])
@pytest.mark.parametrize("top", [16, 32, 33, 64])
@pytest.mark.parametrize("shift", [0, 3])
def test_alternatives_of_short_rows(kernel_set, dtype, vocab, top, shift):
    """As many as a good part of the row's columns, of rows that one wavefront takes, coarse values and so ties among them."""
    x, target, _ = logits(12, vocab, dtype, vocab + top, banned=0.2)
    x[6:] = np.round(x[6:])
    x[11] = np.where(np.arange(vocab) % 64 < 40, -np.inf, x[11])
    pr = Logprob(dtype, x, np.full(12, -1), 1.0, top, pads=(1, 0), shifts=(shift, 0))
    assert pr.fwd(kernel_set) == 0
    sync()
    pr.check_values()


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shift,scale", [(1e30, 1.0), (-1e30, 1.0), (3e4, 30.0), (0.0, 1e-30), (0.0, 1e30)])
def test_large_logits_and_scales(kernel_set, dtype, shift, scale):
    from tests.gpu_util import rnd
    rng = np.random.default_rng(2)
    x = rnd(shift + np.where(np.abs(shift) > 1e20, abs(shift) / 64, 1.0) * rng.normal(0, 1, (4, 700)), dtype)
    pr = Logprob(dtype, x, [0, 5, 699, -1], scale, 3, np.ones(4, np.float32), np.ones(4, np.float32))
    assert pr.fwd(kernel_set) == 0 and pr.bwd(kernel_set) == 0
    sync()
    # log probabilities beyond the largest fp32 number are -inf there
    ref = pr.reference()
    for k in ("logp", "top_logp", "all"):
        ref[k] = np.where(ref[k] < -3.4e38, -np.inf, ref[k])
    pr.check_values(ref)
    if scale < 1e20 and abs(shift) < 1e20:
        pr.check_grad(ref)


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [777, 12000])
def test_in_place_and_again(kernel_set, dtype, vocab):
    """The gradient in the place of the logits, and the same call again: the same bits."""
    import torch
    x, target, (w, dh, dl) = logits(9, vocab, dtype, 3)
    for shift in (0, 1):
        pr = Logprob(dtype, x, target, 0.8, 7, w, dh, dl, (3, 3), (shift, shift))
        assert pr.fwd(kernel_set) == 0 and pr.bwd(kernel_set) == 0
        sync()
        first, kept = pr.dx.clone(), {k: v.clone() for k, v in pr.out.items()}
        assert pr.grad(kernel_set) == 0
        sync()
        second = pr.dx.clone()
        for into in ("bwd", "grad"):
            keep = pr.x.clone()
            assert getattr(pr, into)(kernel_set, into=pr.x) == 0
            sync()
            assert torch.equal(pr.x, first if into == "bwd" else second)
            pr.x.copy_(keep)
        for k, v in pr.out.items():
            assert torch.equal(v, kept[k]), k
        pr.check_grad(dx=second)


@pytest.mark.parametrize("kernel_set", SETS)
def test_outputs_that_are_not_wanted(kernel_set):
    x, target, (w, dh, dl) = logits(5, 3001, "bf16", 4)
    for without in (("logp",), ("stats",), ("entropy",), ("logp", "stats", "entropy")):
        pr = Logprob("bf16", x, target, 1.0, 4)
        assert pr.fwd(kernel_set, without=without) == 0
        sync()
        full = Logprob("bf16", x, target, 1.0, 4)
        assert full.fwd(kernel_set) == 0
        sync()
        for k, v in pr.out.items():
            assert bool(v.isnan().all()) if k in without else bool((v == full.out[k]).all()), k
    pr = Logprob("bf16", x, target, 1.0, 0, w, None, dl)
    assert pr.grad(kernel_set, without=("logp", "entropy")) == 0
    sync()
    pr.check_grad()
    pr = Logprob("bf16", x, None, 1.0, 3)
    assert pr.fwd(kernel_set) == 0
    sync()
    pr.check_values()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cut", [1, 1000, 2999])
def test_a_vocabulary_spread_over_two(dtype, cut):
    """Statistics of two shares joined as their program would, then each share's gradient: what the whole vocabulary's call gives, to the roundings of the joining."""
    import torch
    x, target, (w, dh, dl) = logits(11, 3000, dtype, 8)
    whole = Logprob(dtype, x, target, 0.9, 0, w, dh, dl)
    ref = whole.reference()
    parts = []
    for a, b in ((0, cut), (cut, 3000)):
        here = np.asarray(target) - a
        elsewhere = (np.asarray(target) >= 0) & ((here < 0) | (here >= b - a))
        parts.append(Logprob(dtype, x[:, a:b], here, 0.9, 0, w, dh, dl - np.where(elsewhere, w, 0).astype(np.float32)))
        assert parts[-1].fwd() == 0
    m = torch.maximum(parts[0].out["stats"][:, 0], parts[1].out["stats"][:, 0])
    share = [torch.exp(0.9 * (q.out["stats"][:, 0] - m).double() + q.out["stats"][:, 1].double()) for q in parts]
    ln = torch.log(share[0] + share[1])
    # H = ln S + mean of scale (m - x): each share's mean is its entropy less its own ln S, moved to the common m
    mean = sum(s * (q.out["entropy"] - q.out["stats"][:, 1] + 0.9 * (m - q.out["stats"][:, 0])) for s, q in zip(share, parts)) / (share[0] + share[1])
    got = []
    for q in parts:
        q.out["stats"].copy_(torch.stack((m, ln.float()), 1))
        q.out["entropy"].copy_((ln + mean).float())
        assert q.bwd() == 0
        got.append(q.dx)
    sync()
    whole.check_grad(ref, torch.cat(got, 1))
