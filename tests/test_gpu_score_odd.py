"""Attention of shaped scores on infinities and NaN at lengths of many tiles: what is finite is what the plain kernels, which read nothing but the pairs
that count, say is finite, and it takes a few times what finite inputs take, not a multiple that grows with the length."""
import numpy as np
import pytest

from tests.gpu_util import TOL
from tests.score_util import Attention
from tests.test_gpu_score_attention import inputs, slopes

pytestmark = pytest.mark.gpu
BAD = [float("nan"), float("inf"), float("-inf")]


def results(p):
    return {n: getattr(p, n).float() for n in ("o", "lse", "dq", "dk", "dv")}


@pytest.mark.parametrize("dtype,kernel_set", [("fp32", 0)] + [("bf16", n) for n in (0, 2, 3, 4, 5, 6, 7)])
@pytest.mark.parametrize("value", BAD)
@pytest.mark.parametrize("hd,h,hkv,cap,bias,packed", [(64, 2, 1, 0.0, 0, 1), (128, 4, 2, 20.0, 1, 0)])
@pytest.mark.parametrize("where", ["q", "k", "v", "do", "kv late", "all early"])
def test_what_is_finite(dtype, kernel_set, value, hd, h, hkv, cap, bias, packed, where):
    import torch
    rows = 700
    t = dict(zip(("q", "k", "v", "do"), inputs(dtype, rows, h, hkv, hd, 149)))
    for name, at in {"kv late": [("k", 645), ("v", 646)], "all early": [(n, 3) for n in t]}.get(where, [(where, 300), (where, 301)]):
        t[name][at, 1::7] = value
    opts = dict(cap=cap, slopes=slopes(h) if bias else None)
    opts.update(dict(starts=[0, 5, 260, 690], n_seq=3, prefixes=[0, 40, 70]) if packed else dict(prefixes=[100]))
    got, want = (Attention(dtype, *t.values(), h, hkv, 1, **opts) for _ in range(2))
    for p, s in ((got, kernel_set), (want, 1)):
        assert p.fwd(s) == 0 and p.bwd(s) == 0
    torch.cuda.synchronize()
    got, want = results(got), results(want)
    for n in want:
        ok = torch.isfinite(want[n])
        bad = ok != torch.isfinite(got[n])
        if n == "lse":                                # a row without any weight may be minus infinity or NaN
            bad &= ok
        assert not bool(bad.any()), (n, int(bad.sum()), bad.nonzero()[:4].tolist())
        assert not bool(ok.any()) or float((got[n] - want[n])[ok].abs().max()) <= TOL[dtype] * float(want[n][ok].abs().max()), n


def once(call):
    """Shortest of five, in ms."""
    import torch
    assert call() == 0
    best = float("inf")
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        assert call() == 0
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [512, 2048])
def test_what_it_takes(dtype, hd, rows):
    """Walking every block once more, with loads of its own and without the tiles' reuse, is 5 to 8 times a pass; redoing rows pair by pair was 50 to 200 times at
    these lengths, growing with them."""
    import torch
    h, hkv = 4, 2
    t = dict(zip(("q", "k", "v", "do"), inputs(dtype, rows, h, hkv, hd, 151)))
    clean = Attention(dtype, *t.values(), h, hkv, 1)
    stream = torch.cuda.current_stream().cuda_stream
    limit = [20.0 * once(lambda: call(0, stream)) for call in (clean.fwd, clean.bwd)]
    for name in t:
        for value in BAD[:2]:
            for at in (0, rows - 1):
                x = {n: a.copy() for n, a in t.items()}
                x[name][at, ::3] = value
                p = Attention(dtype, *x.values(), h, hkv, 1)
                took = [once(lambda: call(0, stream)) for call in (p.fwd, p.bwd)]
                assert took[0] <= limit[0] and took[1] <= limit[1], (name, value, at, took, limit)
