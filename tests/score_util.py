"""Calls of the shaped-score attention and per-head norm / rotation entries on NumPy inputs, and the bounds their results have to keep.

Bounds are elementwise.  Rounding to a type is off by at most U = finfo.eps / 2 of the value; P and dS are rounded once before their
products in bf16 (not at all in fp32), outputs once.  F32 is for everything held in fp32 on the way: exponents of up to 100 whose rounding
(2^-24 of them, 6e-6) becomes a relative error of P, sums of up to 128 products, exp, tanh and reciprocal.  It comes to less than 2^-16 of
the terms' absolute values."""
import ctypes as C

import numpy as np

from oracle import score_oracle as sc
from tests.gpu_util import launches, to_dev, to_np

U = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}
F32 = 2.0 ** -16
DT = {"fp32": 0, "bf16": 1}


def ptr(t):
    return None if t is None else t.data_ptr()


def int_tensor(v):
    import torch
    return None if v is None else torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda:0")


def wide(a, dtype, pad, fill=float("nan")):
    """[rows, n] -> the first n columns of a buffer of n + pad ones whose others hold `fill`"""
    import torch
    rows, n = a.shape
    t = torch.full((rows, n + pad), fill, dtype=torch.float32 if dtype == "fp32" else torch.bfloat16, device="cuda:0")
    t[:, :n] = to_dev(a, dtype)
    return t


class Attention:
    """One problem: `run` calls forward and backward and returns NumPy results; outputs start as NaN."""

    def __init__(self, dtype, q, k, v, do, h, hkv, causal, scale=0.0, cap=0.0, slopes=None, starts=None, prefixes=None, n_seq=1, pads=(0, 0, 0, 0, 0)):
        import torch
        from paper_2507_00217_amd import stage as S
        self.S, self.dtype, self.h, self.hkv, self.rows, self.hd = S, dtype, h, hkv, q.shape[0], q.shape[1] // h
        self.opts = dict(h=h, hkv=hkv, causal=causal, scale=scale, cap=cap, slopes=slopes, starts=starts, prefixes=prefixes, n_seq=n_seq)
        self.np = (q, k, v, do)
        self.q, self.k, self.v, self.do = (wide(a, dtype, p) for a, p in zip((q, k, v, do), pads))
        self.keep = [None if slopes is None else torch.tensor(np.asarray(slopes), dtype=torch.float32, device="cuda:0"), int_tensor(starts), int_tensor(prefixes)]
        self.args = S.ScoreAttention(dtype=DT[dtype], rows=self.rows, n_seq=n_seq, h=h, hkv=hkv, hd=self.hd, causal=int(causal), scale=scale, softcap=cap,
                                     slope=ptr(self.keep[0]), seq_start=ptr(self.keep[1]), prefix=ptr(self.keep[2]))
        self.o_pad = pads[4]
        nan = lambda a, p: wide(np.full(a.shape, np.nan, dtype=np.float32), dtype, p)
        self.o, self.dq, self.dk, self.dv = nan(q, pads[4]), nan(q, pads[4]), nan(k, pads[4]), nan(v, pads[4])
        self.lse = torch.full((h, self.rows), float("nan"), device="cuda:0")
        n = S.lib().stage_kernel_score_attention_bwd_scratch_bytes(C.byref(self.args))
        self.scratch = torch.full((n,), 255, dtype=torch.uint8, device="cuda:0")

    def fwd(self, kernel_set=0, stream=None, lse=True):
        m = lambda t: (ptr(t), t.stride(0))
        return self.S.lib().stage_kernel_score_attention_fwd(C.byref(self.args), *m(self.q), *m(self.k), *m(self.v), *m(self.o), ptr(self.lse) if lse else None,
                                                             kernel_set, stream)

    def bwd(self, kernel_set=0, stream=None):
        m = lambda t: (ptr(t), t.stride(0))
        return self.S.lib().stage_kernel_score_attention_bwd(C.byref(self.args), *m(self.q), *m(self.k), *m(self.v), *m(self.o), ptr(self.lse), *m(self.do),
                                                             *m(self.dq), *m(self.dk), *m(self.dv), ptr(self.scratch), self.scratch.numel(), kernel_set, stream)

    def cols(self, t, n):
        return to_np(t[:, :n])

    def o_for(self, kernel_set, o, ref):
        """The o whose rowsum(dO * o) is the delta that dQ and that dK use: `ref` instead of the kernels' rounded `o` for the rows whose delta the bf16
        kernels sum from the probabilities, blocks of 32 queries that see at most 128 keys; in dK only if it has a launch of its own."""
        rows = np.zeros(self.rows, bool)
        if self.dtype == "bf16" and kernel_set != 1 and all(t.stride(0) % 8 == 0 for t in (self.q, self.k, self.v, self.o)):
            for at, n, pre in sc.sequences(self.rows, self.opts["starts"], self.opts["prefixes"], self.opts["n_seq"]):
                for q0 in range(0, n, 32):
                    end = max(min(q0 + 32, n), pre) if self.opts["causal"] else n
                    rows[at + q0:at + min(q0 + 32, n)] = end <= 128
        one_launch = any("score_bwd" in name for name, _, _ in launches(lambda st: self.bwd(kernel_set, st)))
        dq = np.where(rows[:, None], ref, o)
        return dq, o if one_launch else dq

    def backward(self, kernel_set, o, ref, lse):
        """The oracle's gradients with the delta of `o_for`"""
        q, k, v, do = self.np
        o_dq, o_dk = self.o_for(kernel_set, o, ref)
        g = sc.attention_backward(q, k, v, o_dk, lse, do, **self.opts)
        return {**g, "dq": sc.attention_backward(q, k, v, o_dq, lse, do, **self.opts)["dq"]}

    def check(self, kernel_set=0, f32=F32):
        """Runs both directions and compares with the oracle; the backward's oracle takes the kernel's own lse, and its o where delta comes from
        that.  f32: for scores beyond 100."""
        import torch
        q, k, v, do = self.np
        assert self.fwd(kernel_set) == 0
        torch.cuda.synchronize()
        o, lse = self.cols(self.o, q.shape[1]), to_np(self.lse)
        ref, rlse, mag = sc.attention(q, k, v, **self.opts)
        u = U[self.dtype]
        close("o", o, ref, u * np.abs(ref) + ((u if self.dtype == "bf16" else 0) + f32) * mag)
        close("lse", lse, rlse, f32 * (1.0 + np.abs(rlse)))
        assert self.bwd(kernel_set) == 0
        torch.cuda.synchronize()
        for name, (val, rounded, apart) in self.backward(kernel_set, o, ref, lse).items():
            got = self.cols(getattr(self, name), val.shape[1])
            close(name, got, val, u * np.abs(val) + (u if self.dtype == "bf16" else 0) * rounded + f32 * apart)
        for t, n in ((self.o, q.shape[1]), (self.dq, q.shape[1]), (self.dk, k.shape[1]), (self.dv, v.shape[1])):
            assert bool(torch.isnan(t[:, n:].float()).all())                       # nothing is written beside the columns


def close(name, got, ref, bound):
    """Elementwise; where the reference is NaN (rows of no sequence) so is the untouched output."""
    assert got.shape == ref.shape, name
    out = np.isnan(ref)
    assert np.array_equal(out, np.isnan(got)), (name, "NaN", int((out != np.isnan(got)).sum()), np.argwhere(out != np.isnan(got))[:4].tolist())
    d = np.where(out, 0.0, np.abs(got - ref) - np.where(out, 0.0, bound))
    assert (d <= 1e-30).all(), (name, int((d > 0).sum()), np.unravel_index(np.argmax(d), d.shape), float(d.max()), float(np.nanmax(bound)))
