"""Calls of the entries around a training step on NumPy inputs, and the bounds their results have to keep.

U: a rounding to a type is off by at most finfo.eps / 2 of the value.  E = 2^-24 is that of fp32.  A log probability's z = scale (x - m) is made by three roundings
(the difference, the product, scale times log2 e in base 2), its exponential by an instruction good to 2 E: e^z is off by (4 |z| + 4) E of itself, and
where e^z counts at all, e^z |z| < 1.  The sum S of n of them is a tree of at most L(n) additions one behind the other, L the larger of the plain kernel's
(256 threads) and a tile kernel's, so S is off by (8 + L) E; each of its terms' errors 4 |z| e^z E adds at most 4 n' E for the n' terms near the largest, which is
within 4 E (1 + H), H the entropy, of S.  ln S then is off by (12 + L + 4 H) E, and by 2 E of itself."""
import ctypes as C

import numpy as np

from oracle import step_oracle as st
from tests.gpu_util import to_dev, to_np
from tests.score_util import DT, U, ptr

E = 2.0 ** -24
TINY = 2.0 ** -126           # below this fp32 loses what is left


def chain(vocab):
    return vocab / 256 + 20


def close(what, got, want, bound):
    """Where the reference is not finite the result is the same; elsewhere it is within the bound."""
    got, want, bound = (np.asarray(t, dtype=np.float64) for t in (got, want, bound))
    odd = ~np.isfinite(want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    assert same[odd].all(), (what, got[odd & ~same][:4], want[odd & ~same][:4])
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want)
    bad = ~odd & ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], bound[bad][:4] if bound.shape else bound)


def rows_of(a, dtype, pad, shift):
    """[rows, n] -> the same as columns `shift`.. of a buffer of n + pad + shift ones whose others are NaN"""
    import torch
    rows, n = a.shape
    t = torch.full((rows, n + pad + shift), float("nan"), dtype=torch.float32 if dtype == "fp32" else torch.bfloat16, device="cuda:0")
    t[:, shift:shift + n] = to_dev(a, dtype)
    return t, t[:, shift:shift + n]


class Logprob:
    """One problem: fwd, bwd and grad call the entries and return NumPy results; outputs start as NaN (ids as -7)."""

    def __init__(self, dtype, x, target=None, scale=1.0, top=0, w=None, dh=None, dl=None, pads=(0, 0), shifts=(0, 0)):
        import torch
        from paper_2507_00217_amd import stage as S
        self.S, self.L, self.dtype, (self.rows, self.vocab) = S, S.lib(), dtype, x.shape
        self.whole_x, self.x = rows_of(x, dtype, pads[0], shifts[0])
        self.whole_dx, self.dx = rows_of(np.full(x.shape, np.nan, np.float32), dtype, pads[1], shifts[1])
        f = lambda v: None if v is None else torch.tensor(np.asarray(v), dtype=torch.float32, device="cuda:0")
        self.w, self.dh, self.dl = f(w), f(dh), f(dl)
        self.target = None if target is None else torch.tensor(np.asarray(target), dtype=torch.int32, device="cuda:0")
        self.scale, self.top, self.np = scale, top, (x, target, w, dh, dl)
        self.p = S.TokenLogprob(dtype=DT[dtype], rows=self.rows, vocab=self.vocab, top=top, scale=scale, target=ptr(self.target))
        self.scratch = torch.full((self.L.stage_kernel_token_logprob_scratch_bytes(C.byref(self.p)),), 255, dtype=torch.uint8, device="cuda:0")
        nan = lambda *s: torch.full(s, float("nan"), device="cuda:0")
        self.out = dict(logp=nan(self.rows), stats=nan(self.rows, 2), entropy=nan(self.rows), top_id=torch.full((self.rows, top), -7, dtype=torch.int32, device="cuda:0"),
                        top_logp=nan(self.rows, top))

    def values(self, without=()):
        return [None if k in without else ptr(v) for k, v in self.out.items()] + [ptr(self.scratch), self.scratch.numel()]

    def fwd(self, kernel_set=0, stream=None, without=()):
        return self.L.stage_kernel_token_logprob_fwd(C.byref(self.p), ptr(self.x), self.x.stride(0), *self.values(without), kernel_set, stream)

    def bwd(self, kernel_set=0, stream=None, into=None):
        d = self.dx if into is None else into
        return self.L.stage_kernel_token_logprob_bwd(C.byref(self.p), ptr(self.x), self.x.stride(0), ptr(self.out["stats"]), ptr(self.out["entropy"]), ptr(self.w),
                                                     ptr(self.dh), ptr(self.dl), ptr(d), d.stride(0), kernel_set, stream)

    def grad(self, kernel_set=0, stream=None, into=None, without=()):
        d = self.dx if into is None else into
        return self.L.stage_kernel_token_logprob_grad(C.byref(self.p), ptr(self.x), self.x.stride(0), ptr(self.w), ptr(self.dh), ptr(self.dl), ptr(d), d.stride(0),
                                                      *self.values(without), kernel_set, stream)

    def reference(self):
        x, target, *_ = self.np
        return st.token_logprob(x, np.float64(np.float32(self.scale or 1.0)), target, self.top)

    def errors(self, ref):
        """What ln S, any log probability z - ln S and the entropy may be off by"""
        h, ln = np.nan_to_num(ref["entropy"], posinf=0, neginf=0), np.nan_to_num(ref["stats"][:, 1], posinf=0, neginf=0)
        e_ln = (12 + chain(self.vocab) + 4 * h + 2 * np.abs(ln)) * E
        with np.errstate(invalid="ignore"):
            z = np.nan_to_num(np.abs(ref["all"] + ref["stats"][:, 1:2]), nan=0, posinf=0, neginf=0)
        # H = ln S + T / S: T's terms are off like S's, once more for the factor z
        return e_ln, e_ln[:, None] + 4 * E * z + E * np.abs(np.nan_to_num(ref["all"], nan=0, posinf=0, neginf=0)), 2 * e_ln + (24 + 2 * chain(self.vocab)) * E * h + E

    def check_values(self, ref=None, logp=True):
        ref = ref or self.reference()
        e_ln, e_lp, e_h = self.errors(ref)
        g = {k: to_np(v) for k, v in self.out.items()}
        target, rows = self.np[1], np.arange(self.rows)
        has = np.zeros(self.rows, bool) if target is None else (np.asarray(target) >= 0) & (np.asarray(target) < self.vocab)
        at = np.where(has, target if target is not None else 0, 0)
        if logp:
            close("logp", g["logp"], ref["logp"], np.where(has, e_lp[rows, at], 0))
        bad = np.isnan(ref["stats"][:, 0])
        close("m", g["stats"][~bad, 0], ref["stats"][~bad, 0], 0)
        close("ln S", g["stats"][:, 1], ref["stats"][:, 1], e_ln)
        close("entropy", g["entropy"], ref["entropy"], e_h)
        if self.top:
            assert (g["top_id"] == ref["top_id"]).all(), (g["top_id"][:3], ref["top_id"][:3])
            close("top_logp", g["top_logp"], ref["top_logp"], np.take_along_axis(e_lp, np.maximum(ref["top_id"], 0), 1))
        return ref

    def check_grad(self, ref=None, dx=None):
        x, target, w, dh, dl = self.np
        ref = ref or self.reference()
        scale = np.float64(np.float32(self.scale or 1.0))
        f = lambda v: None if v is None else np.asarray(v, np.float32).astype(np.float64)
        want = st.token_logprob_grad(ref["all"], ref["entropy"], scale, target, f(w), f(dh), f(dl), ref["stats"][:, 0] == -np.inf)
        e_ln, e_lp, e_h = self.errors(ref)
        p = np.nan_to_num(np.exp(ref["all"]), nan=0)
        col = lambda v: np.zeros((self.rows, 1)) if v is None else np.abs(f(v))[:, None]
        h = np.nan_to_num(ref["entropy"], posinf=0, neginf=0)[:, None]
        lp = np.abs(np.nan_to_num(ref["all"], nan=0, posinf=0, neginf=0))
        # p is off by e_lp + 4 E of itself, the factor behind it by 4 roundings and by the errors of logp and H, the target's difference by a rounding of what it is of
        mag = col(dl) + col(w) + col(dh) * (lp + h)
        bound = p * (mag * (e_lp + 12 * E) + col(dh) * (e_lp + e_h[:, None])) + 2 * TINY * (1 + mag)
        if target is not None:
            r = np.flatnonzero((np.asarray(target) >= 0) & (np.asarray(target) < self.vocab))
            bound[r, np.asarray(target)[r]] += 2 * E * col(w)[r, 0]
        got = to_np(self.dx if dx is None else dx)
        close("dlogits", got, want, scale * bound + 2 * U[self.dtype] * np.abs(np.nan_to_num(want, nan=0)) + scale * U[self.dtype] * bound)
        return ref


def logits(rows, vocab, dtype, seed, banned=0.0, std=3.0):
    from tests.gpu_util import rnd
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 1, (rows, vocab)) * rng.uniform(0.2, std, (rows, 1)) + rng.normal(0, 4, (rows, 1))
    x = rnd(x, dtype)
    if banned:
        x[rng.random((rows, vocab)) < banned] = -np.inf
    target = rng.integers(0, vocab, rows)
    target[rng.random(rows) < 0.2] = -1
    return x, target, [rng.normal(0, 1, rows).astype(np.float32) for _ in range(3)]
