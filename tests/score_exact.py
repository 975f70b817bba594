"""The shaped-score attention against its definition in 64 bits on the GPU, from the inputs alone: no result of the kernels enters the reference (the
comparison of tests/score_util.py takes the kernels' own lse and o for the backward), and nothing depends on which kernels ran.

Bounds are elementwise and count the stated roundings: outputs once (U), P and dS once before their products (U, bf16), everything else in fp32 (F32 of
tests/score_util.py, once for the scores and once for lse, which is an fp32 result itself).  delta = rowsum(dO * O) takes O as it was stored, which is
off by its own rounding and by that of P: |delta error| <= sum |dO| (U |O| + (U + F32) sum P|V|); a block of 32 queries that sees at most 128 keys has
none of that, since its delta is the sum of P dP.  Products of two of these are below 2^-6 of the whole bound."""
import numpy as np
import torch

from oracle import score_oracle as sc
from tests import score_util
from tests.score_util import U


def definition(p, head, at, n, prefix, exact_delta, F32):
    """One query head of one sequence -> {"o", "lse", "dq", "dk", "dv"}: (value, bound without the output's rounding)."""
    h, hkv, hd, o = p.h, p.hkv, p.hd, p.opts
    u = U[p.dtype] if p.dtype == "bf16" else 0.0
    g = head // (h // hkv)
    col = lambda t, j: t[at:at + n, j * hd:(j + 1) * hd].double()
    q, k, v, do = col(p.q, head), col(p.k, g), col(p.v, g), col(p.do, head)
    scale, cap = o["scale"] or hd ** -0.5, o["cap"]
    s, d = (q @ k.T) * scale, 1.0
    if cap:
        t = torch.tanh(s / cap)
        s, d = cap * t, 1.0 - t * t
    i = torch.arange(n, device=s.device)
    if o["slopes"] is not None:
        s = s - float(np.float32(o["slopes"][head])) * (i[:, None] - i[None, :]).abs()
    if o["causal"]:
        s = s.masked_fill((i[None, :] > i[:, None]) & (i >= prefix)[None, :], -float("inf"))
    lse = torch.logsumexp(s, 1)
    P = torch.softmax(s, 1)                        # (from the differences to the row's highest: s - lse would lose the sum of scores beyond 1e16)
    del s
    out, mag = P @ v, P @ v.abs()
    r = {"o": (out, (u + F32) * mag), "lse": (lse, F32 * (1.0 + lse.abs()))}
    dP, delta = do @ v.T, (do * out).sum(1)
    dS = scale * d * P * (dP - delta[:, None])
    apart = scale * d * P * (do.abs() @ v.abs().T + (do.abs() * out.abs()).sum(1)[:, None])
    block_end = torch.clamp((i // 32 + 1) * 32, max=n) if o["causal"] else torch.full_like(i, n)
    off = (do.abs() * (U[p.dtype] * out.abs() + (u + F32) * mag)).sum(1)
    few = torch.clamp(block_end, min=prefix if o["causal"] else 0) <= 128
    stored = scale * d * P * off[:, None]
    w = u * dS.abs() + 2 * F32 * apart
    wq, wk = (w + torch.where(few[:, None] & flag, 0.0, stored) for flag in exact_delta)
    r["dq"] = (dS @ k, wq @ k.abs())
    r["dk"] = (dS.T @ q, wk.T @ q.abs())
    r["dv"] = (P.T @ do, (u + 2 * F32) * (P.T @ do.abs()))
    return r


def compare(p, groups=None, exact_delta=(True, True), only=None, names=("o", "lse", "dq", "dk", "dv"), rows=None, f32=score_util.F32):
    """p: tests.score_util.Attention after fwd and bwd.  groups: the KV heads to look at.  exact_delta: whether blocks that see few keys have their delta from
    the probabilities in dQ, in dK.  only: predicate on a sequence's length.  names: the results to look at.
    rows: mask of the rows of o, lse and dq to look at.  f32: in the place of F32, for scores beyond 100."""
    dev = lambda b: torch.tensor(b, device=p.q.device)
    flags = tuple(dev(p.dtype == "bf16" and f) for f in exact_delta)
    grp, hd, u = p.h // p.hkv, p.hd, U[p.dtype]
    for g in range(p.hkv) if groups is None else groups:
        for at, n, prefix in sc.sequences(p.rows, p.opts["starts"], p.opts["prefixes"], p.opts["n_seq"]):
            if only is not None and not only(n):
                continue
            kv = {"dk": None, "dv": None}
            span = slice(at, at + n)
            look = torch.ones(n, dtype=torch.bool, device=p.q.device) if rows is None else dev(np.asarray(rows)[span])
            for j in range(g * grp, (g + 1) * grp):
                r = definition(p, j, at, n, prefix, flags, f32)
                for name in kv:
                    kv[name] = r[name] if kv[name] is None else tuple(a + b for a, b in zip(kv[name], r[name]))
                c = slice(j * hd, (j + 1) * hd)
                for name, got in (("o", p.o[span, c]), ("lse", p.lse[j, span]), ("dq", p.dq[span, c])):
                    if name in names:
                        within(name, got[look], *(t[look] for t in r[name]), 0.0 if name == "lse" else u, (j, at))
            c = slice(g * hd, (g + 1) * hd)
            for name, got in (("dk", p.dk[span, c]), ("dv", p.dv[span, c])):
                if name in names:
                    within(name, got, *kv[name], u, (g, at))


def within(name, got, want, bound, u, where):
    d = (got.double() - want).abs() - (1.0 + 2.0 ** -6) * (bound + u * want.abs()) - 1e-30
    assert bool((d <= 0).all()), (name, where, int((~(d <= 0)).sum()), float(d.max()), float(bound.max()))
