"""Attention of shaped scores and per-head norms as programs use them: many sequences, long ones, wide buffers, other streams, captured
graphs, non-finite neighbours, and the operators one behind the other in a layer."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import score_oracle as sc
from oracle import stage_oracle as so
from paper_2507_00217_amd import synth
from tests.gpu_util import TOL, launches, rnd, to_np
from tests.score_util import DT, F32, U, Attention, close, int_tensor, ptr
from tests.test_gpu_score_attention import KERNELS, inputs, slopes

pytestmark = pytest.mark.gpu
ALL = [("fp32", 0)] + [("bf16", n) for n in (0, 2, 3, 4, 5, 6, 7)]


def drawn_lengths(n, rows, seed):
    """n lengths, some of them zero, that add up to rows"""
    rng = np.random.default_rng(seed)
    lens = rng.multinomial(rows, rng.dirichlet(np.full(n, 0.4)))
    return lens


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("n_seq", [64, 65, 200, 5000])
@pytest.mark.parametrize("causal,prefix", [(1, 1), (0, 0)])
def test_many_sequences(dtype, kernel_set, n_seq, causal, prefix):
    """Up to 64 sequences and more than that are found in two ways; many of them are empty."""
    rows, h, hkv, hd = 900, 2, 1, 64
    lens = drawn_lengths(n_seq, rows - 7, n_seq)
    starts = 3 + np.concatenate(([0], np.cumsum(lens)))
    q, k, v, do = inputs(dtype, rows, h, hkv, hd, 71)
    prefixes = [int(n) // 2 for n in lens] if prefix else None
    Attention(dtype, q, k, v, do, h, hkv, causal, starts=starts, prefixes=prefixes, n_seq=n_seq, cap=30.0 if prefix else 0.0).check(kernel_set)


@pytest.mark.parametrize("dtype,kernel_set", ALL)
@pytest.mark.parametrize("hd,cap,prefix", [(64, 0.0, 0), (128, 20.0, 700)])
def test_long_sequence(dtype, kernel_set, hd, cap, prefix):
    rows = 2600
    q, k, v, do = inputs(dtype, rows, 1, 1, hd, 73)
    Attention(dtype, q, k, v, do, 1, 1, 1, cap=cap, slopes=[0.02], prefixes=[prefix]).check(kernel_set)


@pytest.mark.parametrize("dtype,kernel_set", ALL)
def test_large_cap_and_slopes_of_both_signs(dtype, kernel_set):
    """A cap beyond what the forward takes without a running maximum, slopes that raise far keys, and scores far beyond the cap.

    The scores here go past the 100 that F32 is for, so what fp32 may do to a P is counted: an error e of an exponent is a relative error e of P.
    An exponent is made by at most 8 roundings (scale, cap, bias, their sums, lse) of numbers up to M = cap + largest bias + largest |lse|,
    each off by 2^-24 of it; its product q.k by at most 64 roundings of partial sums up to D = scale * sum |q k|, which a cap only shrinks."""
    h, rows, s = 4, 260, [0.5, -0.05, 0.0, -0.3]
    q, k, v, do = inputs(dtype, rows, h, 2, 64, 79, 8.0)
    D = max(float((np.abs(q[:, j * 64:(j + 1) * 64]) @ np.abs(k[:, j // 2 * 64:(j // 2 + 1) * 64]).T).max()) / 8.0 for j in range(h))
    for causal, cap in ((1, 90.0), (0, 25.0)):
        M = cap + 0.5 * rows + (cap + 0.3 * rows + np.log(rows))
        Attention(dtype, q, k, v, do, h, 2, causal, cap=cap, slopes=s).check(kernel_set, f32=2.0 ** -24 * (8 * M + 64 * D))


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_a_sequence_keeps_its_infinities_and_nan(dtype, kernel_set, value):
    """Whatever one sequence holds, the others' results and gradients are the same bits as without it."""
    import torch
    lens, h, hkv, hd = [50, 70, 1, 130], 4, 2, 64
    starts = np.concatenate(([0], np.cumsum(lens)))
    rows = int(starts[-1])
    q, k, v, do = inputs(dtype, rows, h, hkv, hd, 83)
    outs = []
    for bad in (False, True):
        t = [a.copy() for a in (q, k, v, do)]
        if bad:
            for a in t:
                a[starts[1]:starts[2]:3] = value
        p = Attention(dtype, *t, h, hkv, 1, cap=20.0, starts=starts, n_seq=4, prefixes=[5, 5, 0, 200])
        assert p.fwd(kernel_set) == 0 and p.bwd(kernel_set) == 0
        torch.cuda.synchronize()
        outs.append([p.o, p.dq, p.dk, p.dv, p.lse.t()])
    other = torch.ones(rows, dtype=torch.bool, device="cuda:0")
    other[starts[1]:starts[2]] = False
    for a, b in zip(*outs):
        assert bool(torch.isfinite(a[other].float()).all()) and torch.equal(a[other], b[other])


@pytest.mark.parametrize("dtype,kernel_set", ALL)
def test_offsets_beyond_32_bits(dtype, kernel_set):
    """Rows 2^20 elements apart, 2100 of them: the same bits as in compact buffers."""
    import torch
    rows, h, hkv, hd, ld = 2100, 2, 1, 64, 1 << 20
    q, k, v, do = inputs(dtype, rows, h, hkv, hd, 89)
    starts = [0, 30, rows - 3]
    p = Attention(dtype, q, k, v, do, h, hkv, 1, starts=starts, n_seq=2)
    assert p.fwd(kernel_set) == 0 and p.bwd(kernel_set) == 0
    td = torch.float32 if dtype == "fp32" else torch.bfloat16
    big = torch.empty(rows * ld, dtype=td, device="cuda:0").view(rows, ld)
    w = Attention(dtype, q, k, v, do, h, hkv, 1, starts=starts, n_seq=2)
    at = 0
    for n in ("q", "k", "v", "do", "o", "dq", "dk", "dv"):
        t = getattr(w, n)
        view = big[:, at:at + t.shape[1]]
        view.copy_(t)
        setattr(w, n, view)
        at += t.shape[1]
    assert w.fwd(kernel_set) == 0 and w.bwd(kernel_set) == 0
    torch.cuda.synchronize()
    for n in ("o", "dq", "dk", "dv", "lse"):
        a, b = getattr(p, n), getattr(w, n)
        assert torch.equal(torch.nan_to_num(a.float(), 7.0), torch.nan_to_num(b.float(), 7.0)), n
    del big, w


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_forward_without_lse_and_two_streams(dtype):
    """Two problems at once on streams of their own, each with its scratch: what they give one behind the other."""
    import torch
    a, b = (Attention(dtype, *inputs(dtype, rows, 4, 2, 128, seed), 4, 2, 1, cap=cap, n_seq=n) for rows, seed, cap, n in ((700, 91, 0.0, 1), (600, 92, 30.0, 4)))
    ref = []
    for p in (a, b):
        assert p.fwd() == 0 and p.bwd() == 0
        torch.cuda.synchronize()
        ref.append([t.clone() for t in (p.o, p.dq, p.dk, p.dv, p.lse)])
        for t in (p.o, p.dq, p.dk, p.dv, p.lse):
            t.fill_(float("nan"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for p, st in zip((a, b), streams):
            assert p.fwd(stream=st.cuda_stream) == 0 and p.bwd(stream=st.cuda_stream) == 0
    torch.cuda.synchronize()
    for p, r in zip((a, b), ref):
        for x, y in zip((p.o, p.dq, p.dk, p.dv, p.lse), r):
            assert torch.equal(x, y)
    a.o.fill_(0)
    assert a.fwd(lse=False) == 0
    torch.cuda.synchronize()
    assert torch.equal(a.o, ref[0][0])


class Layer:
    """Raw q | k | v -> norm and rotation -> attention -> gradients of all of it, as a layer's attention block runs them: dq, dk and dv land in
    the columns of the projection's gradient, whose first columns the norm's backward then turns into the raw ones in place."""

    def __init__(self, dtype, rows, h, hkv, hd, starts, prefixes, cap, seed=101):
        import torch
        from paper_2507_00217_amd import stage as S
        self.S, self.dtype, self.rows, self.h, self.hkv, self.hd, self.cap = S, dtype, rows, h, hkv, hd, cap
        self.starts, self.prefixes = starts, prefixes
        td = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.td, self.n = td, (h + hkv) * hd
        new = lambda *s: torch.zeros(s, dtype=td, device="cuda:0")
        self.qkv, self.dout = new(rows, (h + 2 * hkv) * hd), new(rows, h * hd)
        self.gamma = new(2, hd)
        rng = np.random.default_rng(seed)
        self.pos = np.stack([np.concatenate([np.arange(b - a) for a, b in zip(starts[:-1], starts[1:])]), rng.integers(0, 30, rows), rng.integers(0, 40, rows)])
        self.section = {64: [8, 12, 12], 128: [16, 24, 24]}[hd]
        self.pos_d, self.starts_d, self.prefix_d = int_tensor(self.pos), int_tensor(starts), int_tensor(prefixes)
        self.axes = S.RopeAxes(n_axes=3, section=tuple(self.section), halves=1, theta=1e4, pos=ptr(self.pos_d), pos_stride=rows)
        self.att = S.ScoreAttention(dtype=DT[dtype], rows=rows, n_seq=len(starts) - 1, h=h, hkv=hkv, hd=hd, causal=1, softcap=cap, seq_start=ptr(self.starts_d),
                                    prefix=ptr(self.prefix_d))
        self.qk, self.rstd, self.o, self.dqkv = new(rows, self.n), torch.zeros(rows, h + hkv, device="cuda:0"), new(rows, h * hd), new(rows, (h + 2 * hkv) * hd)
        self.lse, self.dgamma = torch.zeros(h, rows, device="cuda:0"), torch.zeros(2, hd, device="cuda:0")
        self.part = torch.empty(S.lib().stage_kernel_qk_norm_rope_partial_bytes(hd), dtype=torch.uint8, device="cuda:0")
        self.scratch = torch.empty(S.lib().stage_kernel_score_attention_bwd_scratch_bytes(C.byref(self.att)), dtype=torch.uint8, device="cuda:0")
        self.load(seed)

    def load(self, seed):
        import torch
        f = lambda i, shape, mean=0.0, std=1.0: torch.from_numpy(rnd(synth.normal(seed, i, shape, mean=mean, std=std), self.dtype)).cuda().to(self.td)
        self.qkv.copy_(f(1, tuple(self.qkv.shape), std=1.5))
        self.dout.copy_(f(2, tuple(self.dout.shape)))
        self.gamma.copy_(f(3, tuple(self.gamma.shape), 1.0, 0.2))

    def run(self, stream=None):
        import torch
        L, S, n, d = self.S.lib(), self.S, self.n, self.h * self.hd
        st = torch.cuda.current_stream().cuda_stream if stream is None else stream
        m = lambda t: (ptr(t), t.stride(0))
        q, k, v = self.qk[:, :d], self.qk[:, d:], self.qkv[:, n:]
        dq, dk, dv = self.dqkv[:, :d], self.dqkv[:, d:n], self.dqkv[:, n:]
        self.dgamma.zero_()
        norm = (DT[self.dtype], self.rows, self.h, self.hkv, self.hd)
        g = ptr(self.gamma[0]), ptr(self.gamma[1])
        assert L.stage_kernel_qk_norm_rope_fwd(*norm, 1e-5, C.byref(self.axes), *m(self.qkv), *g, *m(self.qk), ptr(self.rstd), st) == 0
        assert L.stage_kernel_score_attention_fwd(C.byref(self.att), *m(q), *m(k), *m(v), *m(self.o), ptr(self.lse), 0, st) == 0
        assert L.stage_kernel_score_attention_bwd(C.byref(self.att), *m(q), *m(k), *m(v), *m(self.o), ptr(self.lse), *m(self.dout), *m(dq), *m(dk), *m(dv),
                                                  ptr(self.scratch), self.scratch.numel(), 0, st) == 0
        assert L.stage_kernel_qk_norm_rope_bwd(*norm, C.byref(self.axes), *m(self.qkv), ptr(self.rstd), *g, *m(self.dqkv), *m(self.dqkv), ptr(self.dgamma[0]),
                                               ptr(self.dgamma[1]), ptr(self.part), st) == 0

    def results(self):
        return dict(o=self.o, dqkv=self.dqkv, dgamma=self.dgamma)

    def oracle(self):
        qkv, do, gam = to_np(self.qkv), to_np(self.dout), to_np(self.gamma)
        h, hkv, hd, n = self.h, self.hkv, self.hd, self.n
        ang = sc.rope_angles(self.pos, self.section, hd, 1e4, 0)
        w, rstd = sc.qk_norm(qkv[:, :n], gam[0], gam[1], h, hkv, 1e-5)
        qk = sc.rotate(w, ang, hd, 1)
        opts = dict(h=h, hkv=hkv, causal=1, cap=self.cap, starts=self.starts, prefixes=self.prefixes, n_seq=len(self.starts) - 1)
        q, k, v = qk[:, :h * hd], qk[:, h * hd:], qkv[:, n:]
        o, lse, _ = sc.attention(q, k, v, **opts)
        g = sc.attention_backward(q, k, v, o, lse, do, **opts)
        back = sc.rotate(np.concatenate((g["dq"][0], g["dk"][0]), 1), ang, hd, 1, True)
        dx, dgq, dgk = sc.qk_norm_backward(qkv[:, :n], rstd, gam[0], gam[1], h, hkv, back)
        return dict(o=o, dqkv=np.concatenate((dx, g["dv"][0]), 1), dgamma=np.stack((dgq, dgk)))


LAYERS = [("fp32", 230, 4, 2, 64, 0.0), ("bf16", 230, 4, 2, 64, 0.0), ("fp32", 300, 4, 4, 128, 20.0), ("bf16", 700, 8, 2, 128, 20.0)]


@pytest.mark.parametrize("dtype,rows,h,hkv,hd,cap", LAYERS)
def test_attention_block_of_a_layer(dtype, rows, h, hkv, hd, cap):
    """Forward and backward of norm, rotation and attention together, within the whole path's tolerance of the engine (tests/gpu_util.py)."""
    import torch
    starts = [0, rows // 5, rows // 5, rows // 2 + 3, rows]
    layer = Layer(dtype, rows, h, hkv, hd, starts, [3, 0, 40, 0], cap)
    layer.run()
    torch.cuda.synchronize()
    ref = layer.oracle()
    for name, t in layer.results().items():
        assert so.max_rel_err(to_np(t), ref[name]) <= TOL[dtype], name


@pytest.mark.parametrize("dtype,rows,h,hkv,hd,cap", LAYERS[:2] + LAYERS[3:])
def test_captured_attention_block(dtype, rows, h, hkv, hd, cap):
    """The block in a captured graph, replayed with new inputs and eager work in between: every replay the same bits as the eager block."""
    import torch
    starts = [0, rows // 3, rows]
    layer = Layer(dtype, rows, h, hkv, hd, starts, [5, 0], cap)
    layer.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.run()
    for seed in (201, 202, 203, 204):
        layer.load(seed)
        layer.run()
        torch.cuda.synchronize()
        want = {n: t.clone() for n, t in layer.results().items()}
        for t in layer.results().values():
            t.fill_(float("nan"))
        junk = torch.randn(500, 500, device="cuda:0") @ torch.randn(500, 500, device="cuda:0")
        graph.replay()
        torch.cuda.synchronize()
        assert bool(torch.isfinite(junk).all())
        for n, t in layer.results().items():
            assert torch.equal(t, want[n]), (seed, n)


def test_the_rules_reach_every_kernel():
    """Every form of the bf16 kernels is what some sizes get without asking for it (read off a stream capture, nothing runs)."""
    import re

    import torch
    from paper_2507_00217_amd import stage as S
    buf = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda:0")
    starts = torch.zeros(1 << 12, dtype=torch.int32, device="cuda:0")
    seen = set()
    for hd in (64, 128):
        for cap in (0.0, 30.0):
            for rows, n_seq, h, hkv, packed in [      # (rows < 0: so many without a causal mask)
                                                (8192, 1, 32, 32, 0), (4096, 2, 32, 8, 0), (8192, 13, 16, 2, 1), (2048, 1, 16, 16, 0), (5000, 1, 4, 4, 0), (2400, 3, 12, 12, 0),
                                                (600, 6, 8, 8, 1), (8192, 100, 16, 16, 1), (1024, 1, 8, 8, 0), (9000, 1, 12, 12, 0), (6000, 5, 8, 8, 1), (700, 1, 40, 40, 0),
                                                (3000, 1, 16, 16, 0), (6000, 1, 6, 6, 0), (1000, 5, 12, 12, 0), (-2048, 1, 8, 8, 0),
                                                (900, 3, 8, 8, 0), (300, 1, 36, 36, 0)]:
                a = S.ScoreAttention(dtype=1, rows=abs(rows), n_seq=n_seq, h=h, hkv=hkv, hd=hd, causal=int(rows > 0), softcap=cap, seq_start=starts.data_ptr() if packed else None)
                p, d, dk = buf.data_ptr(), h * hd, hkv * hd
                need = S.lib().stage_kernel_score_attention_bwd_scratch_bytes(C.byref(a))
                m = (p, d, p, dk, p, dk, p, d)
                for name, _, _ in launches(lambda st: S.lib().stage_kernel_score_attention_fwd(C.byref(a), *m, p, 0, st)):
                    seen.add(name)
                for name, _, _ in launches(lambda st: S.lib().stage_kernel_score_attention_bwd(C.byref(a), *m, p, p, d, p, d, p, dk, p, dk, p, need, 0, st)):
                    seen.add(name)
    forms = {re.sub(r".*?score_(\w+?)_kernelI(.*?)EEEvNS.*", r"\1 \2", n) for n in seen if "score_" in n and "reduce" not in n}
    want = set()
    for hd in (64, 128):
        for cap in (0, 1):
            fwd = ["512ELi1", "256ELi1", "256ELi2", "512ELi4"] if hd == 128 else ["256ELi1", "256ELi2", "512ELi4"]
            want |= {f"fwd Li{hd}ELi{f}ELb{cap}" for f in fwd}
            want |= {f"dq Li{hd}ELi{f}ELb{cap}" for f in ("512ELi1", "256ELi1", "256ELi2")}
            want |= {f"dkv Li{hd}ELi{f}ELb{cap}" for f in ("128ELi1", "64ELi1", "64ELi2")}
            want |= {f"bwd Li{hd}ELi{f}ELb{cap}" for f in ("4ELi2", "2ELi1")}
    assert forms == want, (sorted(want - forms), sorted(forms - want))


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("hd,cap,h,hkv", [(64, 0.0, 2, 2), (128, 20.0, 4, 1)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", ["keys", "queries"])
def test_nothing_behind_the_mask_reaches_a_row(dtype, kernel_set, hd, cap, h, hkv, value, where):
    """An infinity or NaN in the keys and values of one row (or in its query and dO): what does not see it is what it is without.  Row 85 lies
    inside a block of 32, so its tile is shared with rows on both sides; the prefix of 20 keys does not hold it."""
    import torch
    rows, r = 150, 85
    q, k, v, do = inputs(dtype, rows, h, hkv, hd, 97)
    bad = [a.copy() for a in (q, k, v, do)]
    for a in (bad[1:3] if where == "keys" else (bad[0], bad[3])):
        a[r, 1::5] = value
    p = Attention(dtype, *bad, h, hkv, 1, cap=cap, prefixes=[20])
    assert p.fwd(kernel_set) == 0 and p.bwd(kernel_set) == 0
    torch.cuda.synchronize()
    o, lse = to_np(p.o), to_np(p.lse)
    rest = np.arange(rows) < r if where == "keys" else np.arange(rows) != r       # rows of o and dq that do not see it
    after = np.arange(rows) > r                                                  # keys that no such query sees
    opts = p.opts
    ref, rlse, mag = sc.attention(q, k, v, **opts)
    u = U[dtype]
    lo = u if dtype == "bf16" else 0.0
    close("o", o[rest], ref[rest], u * np.abs(ref[rest]) + (lo + F32) * mag[rest])
    close("lse", lse[:, rest], rlse[:, rest], F32 * (1.0 + np.abs(rlse[:, rest])))
    o = np.where(rest[:, None], o, ref)
    lse = np.where(rest[None], lse, rlse)
    p.np = (q, k, v, do)
    g = p.backward(kernel_set, o, ref, lse)
    for name in ("dq",) if where == "keys" else ("dq", "dk", "dv"):
        part = rest if name == "dq" else after
        val, rounded, apart = (t[part] for t in g[name])
        close(name, to_np(getattr(p, name))[part], val, u * np.abs(val) + lo * rounded + F32 * apart)
    seen = ~rest if where == "keys" else np.arange(rows) == r
    assert np.isnan(to_np(p.o)[seen]).any(1).all() or not math.isnan(value)      # and what does see a NaN is NaN


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("n_seq", [2, 70])
@pytest.mark.parametrize("first", [20, 150, 330])
def test_sequences_that_start_late(dtype, kernel_set, n_seq, first):
    """Many rows before the first sequence: more than a workgroup's, and all but a few."""
    rows, h, hkv, hd = 400, 2, 1, 64
    q, k, v, do = inputs(dtype, rows, h, hkv, hd, 103)
    starts = first + np.concatenate(([0], np.cumsum(drawn_lengths(n_seq, rows - first - 1, n_seq))))
    Attention(dtype, q, k, v, do, h, hkv, 1, starts=starts, n_seq=n_seq, cap=20.0, slopes=[0.01, 0.1]).check(kernel_set)


@pytest.mark.parametrize("dtype,kernel_set", KERNELS)
@pytest.mark.parametrize("n_seq", [5, 90])
def test_disordered_offsets_stay_inside_the_rows(dtype, kernel_set, n_seq):
    """Offsets out of order, negative or beyond the rows, and prefixes likewise: nothing outside the rows is written, and the next call with good
    ones is right.  (Every buffer lies between rows of its own, so that a stray access would find memory that belongs to the test.)"""
    import torch
    rows, h, hkv, hd, guard = 300, 2, 1, 64, 512
    q, k, v, do = inputs(dtype, rows, h, hkv, hd, 101)
    rng = np.random.default_rng(n_seq)
    starts = rng.integers(-2 * rows, 3 * rows, n_seq + 1)
    starts[:3] = (-2 ** 31, 2 ** 31 - 1, 40)
    p = Attention(dtype, q, k, v, do, h, hkv, 1, starts=starts, prefixes=rng.integers(-2 * rows, 2 * rows, n_seq), n_seq=n_seq, cap=20.0, slopes=[0.01, 0.1])
    around = {}
    for n in ("q", "k", "v", "do", "o", "dq", "dk", "dv"):
        t = getattr(p, n)
        around[n] = torch.full((rows + 2 * guard, t.shape[1]), float("nan"), dtype=t.dtype, device="cuda:0")
        around[n][guard:guard + rows] = t
        setattr(p, n, around[n][guard:guard + rows])
    flat = torch.full((h * rows + 2 * guard,), float("nan"), device="cuda:0")
    p.lse = flat[guard:guard + h * rows].view(h, rows)
    space = torch.full((p.scratch.numel() + 2 * guard,), 90, dtype=torch.uint8, device="cuda:0")
    p.scratch = space[guard:guard + p.scratch.numel()]
    assert p.fwd(kernel_set) == 0 and p.bwd(kernel_set) == 0
    torch.cuda.synchronize()
    for t in around.values():
        assert bool(torch.isnan(t[:guard].float()).all()) and bool(torch.isnan(t[guard + rows:].float()).all())
    assert bool(torch.isnan(flat[:guard]).all()) and bool(torch.isnan(flat[-guard:]).all())
    assert bool((space[:guard] == 90).all()) and bool((space[-guard:] == 90).all())
    Attention(dtype, q, k, v, do, h, hkv, 1, starts=[0, 100, rows], n_seq=2, cap=20.0, slopes=[0.01, 0.1]).check(kernel_set)
