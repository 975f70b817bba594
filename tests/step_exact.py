"""Log probabilities, entropy and the logits' gradient in 64 bits on the GPU, whole rows at once, and what fp32 kernels may be off by.

E = 2^-24 is fp32's rounding.  With z = scale (x - m) natural exponents, t = sum p |z| and q = sum p z^2 of a row:
  a term e^z is made by three roundings of its exponent (the difference, the constant, the product) and one more where it is taken against another base, and an instruction good to 2 E: off by
  (4 |z| + 2) E of itself; a sum S of terms of one sign that are added `chain` times one behind the other by (chain + 2 + 4 t) E of itself, and the logarithm by 2 E of its own size:
    ln S: (12 + chain + 4 t + 2 |ln S|) E;   z - ln S: that, 4 |z| E, and E of itself
  T = sum of e^z |z|: its terms by the exponential's error and four roundings, its quotient with S by that of S besides:
    H = ln S + T / S: ln S's, (4 q + (12 + 2 chain + 4 t) t) E, and three roundings
  p = e^(z - ln S): ln S's, and its exponent's roundings (4 |z| + 2 |ln p| + 3 |ln S| + 4) E; the factor behind it eight roundings of its terms' sizes and, with the entropy's weight, the errors
  of ln p and H; the token's weight two roundings and the sum's one."""
import math

import numpy as np
import torch

E = 2.0 ** -24
U = {torch.float32: torch.finfo(torch.float32).eps / 2, torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2}
LEAST = 2.0 ** -126               # the exponential of fp32 gives nothing below it


class Rows:
    def __init__(self, x, scale, target, chain):
        self.x, self.scale, self.dtype = x, float(np.float32(scale or 1.0)), x.dtype
        x = x.double()
        self.bad = (torch.isnan(x) | (x == math.inf)).any(1)
        self.empty = (x == -math.inf).all(1)
        odd = (self.bad | self.empty)[:, None]
        x = torch.where(odd, 0.0, x)
        self.m = x.amax(1)
        z = (x - self.m[:, None]) * self.scale
        e = torch.exp(z)
        total = e.sum(1)
        self.ln = torch.log(total)
        self.lp = z - self.ln[:, None]
        self.p = e / total[:, None]
        self.az = torch.where(e > 0, -z, 0.0)
        t, q = (self.p * self.az).sum(1), (self.p * self.az ** 2).sum(1)
        self.h = self.ln + t
        self.e_ln = (12 + chain + 4 * t + 2 * self.ln) * E
        self.e_h = self.e_ln + (4 * q + (12 + 2 * chain + 4 * t) * t + 3 * (self.ln + t) + 1) * E
        self.has = torch.zeros_like(self.bad) if target is None else (target >= 0) & (target < x.shape[1])
        self.at = torch.where(self.has, 0 if target is None else target, 0).long()

    def _rows(self, got, want, bound, bad, empty, what):
        """bad rows are NaN, rows of nothing but -inf are `empty`, others within the bound"""
        got = got.double()
        assert bool(torch.isnan(got[self.bad]).all()) if bad is None else bool((got[self.bad] == bad).all()), what
        assert bool((got[self.empty] == empty).all()), what
        ok = ~(self.bad | self.empty)
        off = (got - want).abs()
        worse = ~(off <= bound) & (ok if off.dim() == 1 else ok[:, None])
        assert not bool(worse.any()), (what, int(worse.sum()), worse.nonzero()[:4].tolist(), got[worse][:4].tolist(), want[worse][:4].tolist())

    def check_values(self, logp=None, stats=None, entropy=None):
        if stats is not None:
            ok = ~(self.bad | self.empty)
            assert torch.equal(stats[ok, 0].double(), self.m[ok]) and bool((stats[self.empty, 0] == -math.inf).all())
            self._rows(stats[:, 1], self.ln, self.e_ln, None, -math.inf, "ln S")
        if entropy is not None:
            self._rows(entropy, self.h, self.e_h, None, 0.0, "entropy")
        if logp is not None:
            assert bool((logp[~self.has] == 0).all())
            take = lambda v: v.gather(1, self.at[:, None])[:, 0]
            lp, az = take(self.lp), take(self.az)
            gone = self.has & ~(self.bad | self.empty) & torch.isinf(lp)          # a token that cannot be
            assert bool((logp[gone] == -math.inf).all())
            keep = self.has & ~gone
            same = self.bad & keep
            assert bool(torch.isnan(logp[same]).all()) and bool((logp[self.empty & keep] == -math.inf).all())
            keep = keep & ~(self.bad | self.empty)
            off, bound = (logp.double() - lp).abs(), self.e_ln + (4 * az + lp.abs()) * E
            assert bool((off[keep] <= bound[keep]).all()), ("logp", off[keep].max())

    def check_grad(self, dx, w=None, dh=None, dl=None):
        zero = torch.zeros_like(self.ln)
        w = zero if w is None else torch.where(self.has, w.double(), 0.0)
        dh, dl = (zero if v is None else v.double() for v in (dh, dl))
        none = (w == 0) & (dh == 0) & (dl == 0)
        assert bool((dx[none | self.empty] == 0).all())
        col = lambda v: v[:, None]
        seen = self.p > 0
        lp = torch.where(seen, self.lp, 0.0)
        want = torch.where(seen, self.p * (col(dl - w) - col(dh) * (lp + col(self.h))), 0.0)
        mag = col(dl.abs() + w.abs()) + col(dh.abs()) * (lp.abs() + col(self.h))
        e_lp = col(self.e_ln) + (4 * self.az + lp.abs()) * E
        e_p = col(self.e_ln) + (4 * self.az + 2 * lp.abs() + 3 * col(self.ln) + 4) * E
        bound = self.p * (mag * (e_p + 8 * E) + col(dh.abs()) * (e_lp + col(self.e_h))) + 2 * LEAST * (1 + mag)
        here = col(self.at)
        want.scatter_add_(1, here, col(w))
        bound.scatter_add_(1, here, col(3 * E * w.abs()))
        want, bound = want * self.scale, bound * self.scale
        bound = bound + U[self.dtype] * (want.abs() + bound) + E * want.abs()
        got = dx.double()
        live = ~(none | self.empty)
        assert bool(torch.isnan(got[self.bad & live]).all()), "rows that are not finite"
        live = live & ~self.bad
        worse = ~((got - want).abs() <= bound) & live[:, None]
        assert not bool(worse.any()), (int(worse.sum()), worse.nonzero()[:4].tolist(), got[worse][:4].tolist(), want[worse][:4].tolist(), bound[worse][:4].tolist())
