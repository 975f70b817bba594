"""What surrounds a stage in a training step, written out in NumPy fp64 (include/stage_kernels.h has the definitions in words): log probabilities of the
rows' tokens with entropy, alternatives and the logits' gradient; the norm of many gradients and the clip to a largest one; the AdamW step."""
from __future__ import annotations

import math

import numpy as np


def token_logprob(x, scale=1.0, target=None, top=0):
    """x: [rows, vocab] -> {logp, stats, entropy, top_id, top_logp, all} (all: the log probability of every column)"""
    rows, vocab = x.shape
    out = dict(logp=np.zeros(rows), stats=np.empty((rows, 2)), entropy=np.empty(rows), top_id=np.empty((rows, top), dtype=np.int64),
               top_logp=np.empty((rows, top)), all=np.empty((rows, vocab)))
    for r in range(rows):
        v = x[r].astype(np.float64)
        order = sorted(range(vocab), key=lambda j: (-v[j], j))[:top] if top else []
        if np.isnan(v).any() or (v == np.inf).any():
            logp, m, ln, h, order = np.full(vocab, np.nan), np.nan, np.nan, np.nan, [-1] * top
        elif (v == -np.inf).all():
            logp, m, ln, h = np.full(vocab, -np.inf), -np.inf, -np.inf, 0.0
        else:
            m = v.max()
            z = scale * (v - m)
            ln = math.log(np.exp(z).sum())
            logp = z - ln
            seen = np.exp(logp) > 0
            h = -(np.exp(logp[seen]) * logp[seen]).sum()
        out["all"][r], out["stats"][r], out["entropy"][r] = logp, (m, ln), h
        out["top_id"][r] = order
        out["top_logp"][r] = [logp[j] for j in order]
        if target is not None and 0 <= target[r] < vocab:
            out["logp"][r] = logp[target[r]]
    return out


def token_logprob_grad(logp, entropy, scale=1.0, target=None, dlogp=None, dentropy=None, dlse=None, empty=None):
    """From the log probability of every column (of these columns, where the vocabulary is wider) -> dlogits; empty: rows without a distribution"""
    rows, vocab = logp.shape
    g = np.zeros((rows, vocab))
    for r in range(rows):
        t = target[r] if target is not None and 0 <= target[r] < vocab else None
        w = float(dlogp[r]) if dlogp is not None and t is not None else 0.0
        dh = float(dentropy[r]) if dentropy is not None else 0.0
        dl = float(dlse[r]) if dlse is not None else 0.0
        if (w == 0.0 and dh == 0.0 and dl == 0.0) or (empty is not None and empty[r]):
            continue
        p = np.exp(logp[r])
        with np.errstate(invalid="ignore"):
            g[r] = np.where(p == 0.0, 0.0, p * (dl - w - dh * (np.where(p == 0.0, 0.0, logp[r]) + (entropy[r] if dh else 0.0))))
        if t is not None:
            g[r, t] += w
    return scale * g


def sumsq(tensors):
    return math.fsum(float(v) ** 2 for t in tensors for v in np.asarray(t, dtype=np.float64).ravel())


def clip_factor(total, max_norm):
    norm = math.sqrt(total) if total == total else total
    return max_norm / norm if norm > max_norm and math.isfinite(norm) else 1.0


def adamw(w, m, v, g, lr, beta1, beta2, eps, weight_decay, step):
    """-> (w, m, v)"""
    w, m, v, g = (np.asarray(t, dtype=np.float64) for t in (w, m, v, g))
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    return w - lr * (weight_decay * w + m / (1.0 - beta1 ** step) / (np.sqrt(v / (1.0 - beta2 ** step)) + eps)), m, v
