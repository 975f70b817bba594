"""Rotary positions on several axes, per-head norms of queries and keys, and attention of shaped scores over packed
sequences, written out step by step in NumPy fp64 (include/stage_kernels.h has the definitions in words).

Rows are [rows, heads * hd] as the engine stores them; every backward is the formula, not automatic differentiation.
"""
from __future__ import annotations

import math

import numpy as np


def rope_angles(pos, section, hd, theta, restart):
    """[rows, hd/2] angles; pos: [axes, rows] integers."""
    cols, first = [], 0
    for axis, n in enumerate(section):
        q = np.arange(n, dtype=np.float64)
        freq = float(theta) ** (-(q / n) if restart else -2.0 * (first + q) / hd)
        cols.append(np.asarray(pos[axis], dtype=np.float64)[:, None] * freq)
        first += n
    assert first == hd // 2
    return np.concatenate(cols, 1)


def rotate(x, angles, hd, halves, inverse=False):
    """x: [rows, heads * hd]"""
    v = x.astype(np.float64).reshape(x.shape[0], -1, hd)
    a, b = (v[..., :hd // 2], v[..., hd // 2:]) if halves else (v[..., 0::2], v[..., 1::2])
    c, s = np.cos(angles)[:, None, :], np.sin(angles)[:, None, :] * (-1.0 if inverse else 1.0)
    ra, rb = a * c - b * s, a * s + b * c
    out = np.empty_like(v)
    if halves:
        out[..., :hd // 2], out[..., hd // 2:] = ra, rb
    else:
        out[..., 0::2], out[..., 1::2] = ra, rb
    return out.reshape(x.shape)


def _gammas(gq, gk, h, hkv):
    return np.concatenate((np.repeat(gq[None].astype(np.float64), h, 0), np.repeat(gk[None].astype(np.float64), hkv, 0)))


def qk_norm(x, gq, gk, h, hkv, eps):
    """x: [rows, (h + hkv) * hd] -> (normalised and weighted, not yet rotated; rstd [rows, h + hkv])"""
    v = x.astype(np.float64).reshape(x.shape[0], h + hkv, -1)
    rstd = 1.0 / np.sqrt((v * v).mean(-1) + eps)
    return (v * rstd[..., None] * _gammas(gq, gk, h, hkv)).reshape(x.shape), rstd


def qk_norm_backward(x, rstd, gq, gk, h, hkv, g):
    """g: gradient of the normalised and weighted heads (already rotated back) -> (dx, dgq, dgk)"""
    hd = x.shape[1] // (h + hkv)
    v, g = (t.astype(np.float64).reshape(-1, h + hkv, hd) for t in (x, g))
    n = v * rstd.astype(np.float64)[..., None]
    dg = (g * n).sum(0)
    gw = g * _gammas(gq, gk, h, hkv)
    dx = rstd[..., None] * (gw - n * (gw * n).mean(-1, keepdims=True))
    return dx.reshape(x.shape), dg[:h].sum(0), dg[h:].sum(0)


def visible(n, causal, prefix):
    """[n, n]: whether query i of a sequence sees its key j"""
    i = np.arange(n)
    return (i[None, :] <= i[:, None]) | (i < prefix)[None, :] if causal else np.ones((n, n), dtype=bool)


def _scores(q, k, scale, cap, slope):
    """(scores, derivative of the cap)"""
    s = scale * (q @ k.T)
    d = np.ones_like(s)
    if cap > 0:
        t = np.tanh(s / cap)
        s, d = cap * t, 1.0 - t * t
    i = np.arange(len(q))
    return s - slope * np.abs(i[:, None] - i[None, :]), d


def _head(a, j, hd):
    return a[:, j * hd:(j + 1) * hd].astype(np.float64)


def sequences(rows, starts, prefixes, n_seq):
    """(first row, rows, prefix) of every sequence that has any"""
    if starts is None:
        starts = np.arange(n_seq + 1) * (rows // n_seq)
    for i in range(n_seq):
        n = int(starts[i + 1] - starts[i])
        if n:
            yield int(starts[i]), n, 0 if prefixes is None else min(max(int(prefixes[i]), 0), n)


def attention(q, k, v, h, hkv, causal, scale=0.0, cap=0.0, slopes=None, starts=None, prefixes=None, n_seq=1):
    """(o, lse, sum_j p_ij |v_j|); rows of no sequence are NaN.  The third is what the rounding of p to a narrower type is measured by."""
    rows, hd = q.shape[0], q.shape[1] // h
    scale = scale or 1.0 / math.sqrt(hd)
    o, mag = np.full((rows, h * hd), np.nan), np.full((rows, h * hd), np.nan)
    lse = np.full((h, rows), np.nan)
    for at, n, pre in sequences(rows, starts, prefixes, n_seq):
        r, seen = slice(at, at + n), visible(n, causal, pre)
        for j in range(h):
            g = j // (h // hkv)
            s, _ = _scores(_head(q[r], j, hd), _head(k[r], g, hd), scale, cap, 0.0 if slopes is None else float(slopes[j]))
            s = np.where(seen, s, -np.inf)
            m = s.max(1)
            p = np.exp(s - m[:, None])
            l = p.sum(1)
            c = slice(j * hd, (j + 1) * hd)
            vg = _head(v[r], g, hd)
            o[r, c], lse[j, r], mag[r, c] = (p / l[:, None]) @ vg, m + np.log(l), (p / l[:, None]) @ np.abs(vg)
    return o, lse, mag


def attention_backward(q, k, v, o, lse, do, h, hkv, causal, scale=0.0, cap=0.0, slopes=None, starts=None, prefixes=None, n_seq=1):
    """Gradients from the forward's o and lse as they are handed over: {"dq", "dk", "dv"}, each (value, sums of the absolute values of what
    it is a sum of when the factor P or dS is rounded, the same with dP and delta taken apart); rows of no sequence are NaN."""
    rows, hd = q.shape[0], q.shape[1] // h
    scale = scale or 1.0 / math.sqrt(hd)
    out = {n: tuple(np.full(t.shape, np.nan) for _ in range(3)) for n, t in (("dq", q), ("dk", k), ("dv", v))}
    for at, n, pre in sequences(rows, starts, prefixes, n_seq):
        r, seen = slice(at, at + n), visible(n, causal, pre)
        for name in ("dk", "dv"):
            for t in out[name]:
                t[r] = 0.0
        for j in range(h):
            g = j // (h // hkv)
            qj, kg, vg, dj, oj = _head(q[r], j, hd), _head(k[r], g, hd), _head(v[r], g, hd), _head(do[r], j, hd), _head(o[r], j, hd)
            s, d = _scores(qj, kg, scale, cap, 0.0 if slopes is None else float(slopes[j]))
            p = np.where(seen, np.exp(np.where(seen, s, -np.inf) - lse[j, r].astype(np.float64)[:, None]), 0.0)
            ds = scale * d * p * (dj @ vg.T - (dj * oj).sum(1)[:, None])
            apart = scale * d * p * (np.abs(dj) @ np.abs(vg).T + (np.abs(dj) * np.abs(oj)).sum(1)[:, None])
            c, cg = slice(j * hd, (j + 1) * hd), slice(g * hd, (g + 1) * hd)
            for t, w in zip(out["dq"], (ds, np.abs(ds), apart)):
                t[r, c] = w @ (kg if w is ds else np.abs(kg))
            for t, w in zip(out["dk"], (ds, np.abs(ds), apart)):
                t[r, cg] += w.T @ (qj if w is ds else np.abs(qj))
            for t, x in zip(out["dv"], (dj, np.abs(dj), np.abs(dj))):
                t[r, cg] += p.T @ x
    return out
