"""The entries around a training step as programs use them: a pipeline's last stage with its head, loss and update; captured graphs, other streams, long rows and lists,
offsets beyond 32 bits; and which kernels the rules come to."""
import ctypes as C
import math
import re

import numpy as np
import pytest

from oracle import stage_oracle as so
from oracle import step_oracle as st
from paper_2507_00217_amd import synth
from tests.gpu_util import SMALL, TOL, launches, rnd, shape_of, to_dev, to_np
from tests.score_util import DT, ptr
from tests.step_util import E, Logprob, logits
from tests.test_gpu_grad_update import List, Update, sumsq, values

pytestmark = pytest.mark.gpu


def sync():
    import torch
    torch.cuda.synchronize()


# ---------------------------------------------------------------------------
# the last stage of a pipeline, one iteration
# ---------------------------------------------------------------------------
FP32 = dict(synth.CONFIGS["cfg1"], hidden=256, n_heads=4, n_kv_heads=2, ffn=512, seq=96)


@pytest.mark.parametrize("cfg,vocab", [(FP32, 1003), (SMALL["cfg3s"], 4001), (SMALL["cfg2s"], 2048)])
def test_an_iteration_of_the_last_stage(cfg, vocab):
    """F of every microbatch, the head's product, the loss with its gradient, the head's products back, B and W; then the norm over stage and head, and the update of both.
    Gradients against the oracle within the whole path's tolerance (tests/gpu_util.py); the update against its formula, from the gradients as they are."""
    import torch
    from paper_2507_00217_amd import stage as S
    dtype, d, n_mb, rows = cfg["dtype"], cfg["hidden"], 2, cfg["mb_size"] * cfg["seq"]
    cfg = dict(cfg, n_microbatches=n_mb, stash_cap=0)
    L, td = S.lib(), torch.float32 if dtype == "fp32" else torch.bfloat16
    rng = np.random.default_rng(9)
    params, X = synth.make_weights(cfg, 31), synth.make_boundary(cfg, 32)
    pad = -vocab % 8                                     # the head's columns are padded to whole 16 bytes; the loss sees the vocabulary
    head = rnd(np.concatenate((rng.normal(0, 0.05, (d, vocab)), np.zeros((d, pad))), 1), dtype)
    target = rng.integers(-1, vocab, (n_mb, rows))
    stage = S.Stage(cfg)
    stage.load_weights(params)
    Xd, Wh, dWh = to_dev(X, dtype).view(n_mb, rows, d), to_dev(head, dtype), torch.zeros(d, vocab + pad, device="cuda:0")
    Y, dY, dX = (torch.zeros_like(Xd) for _ in range(3))
    w = torch.full((rows,), -1.0 / (n_mb * rows), device="cuda:0")
    tg = torch.tensor(target, dtype=torch.int32, device="cuda:0")
    logp, stats = torch.zeros(n_mb, rows, device="cuda:0"), torch.zeros(rows, 2, device="cuda:0")
    i64 = C.c_int64
    gemm = lambda mode, M, N, K, A, lda, B, ldb, Cm, ldc, acc: L.stage_kernel_gemm(DT[dtype], mode, M, N, K, C.c_void_p(ptr(A)), i64(lda), C.c_void_p(ptr(B)), i64(ldb),
                                                                                   C.c_void_p(ptr(Cm)), i64(ldc), None, i64(0), acc, 0, None)
    n = vocab + pad
    for mb in range(n_mb):
        stage.forward(mb, Xd[mb], Y[mb])
        x = torch.empty(rows, n, dtype=td, device="cuda:0")
        assert gemm(0, rows, n, d, Y[mb], d, Wh, n, x, n, 0) == 0
        p = S.TokenLogprob(dtype=DT[dtype], rows=rows, vocab=vocab, top=0, scale=1.0, target=ptr(tg[mb]))
        scratch = torch.empty(L.stage_kernel_token_logprob_scratch_bytes(C.byref(p)), dtype=torch.uint8, device="cuda:0")
        x[:, vocab:] = 0                                 # the gradient takes the logits' place; what lies behind it is zero for the products
        assert L.stage_kernel_token_logprob_grad(C.byref(p), ptr(x), n, ptr(w), None, None, ptr(x), n, ptr(logp[mb]), ptr(stats), None, None, None, ptr(scratch), scratch.numel(), 0, None) == 0
        assert gemm(1, rows, d, n, x, n, Wh, n, dY[mb], d, 0) == 0 and gemm(2, d, n, rows, Y[mb], d, x, n, dWh, n, 1) == 0
        stage.backward_input(mb, dY[mb], dX[mb])
    for mb in range(n_mb):
        stage.backward_weight(mb)
    sync()
    # the oracle
    ref = so.OracleStage(shape_of(cfg), params)
    lay = (cfg["mb_size"], cfg["seq"], d)
    ref_dwh = np.zeros((d, vocab))
    hv = head[:, :vocab].astype(np.float64)
    for mb in range(n_mb):
        y = ref.forward(mb, X[mb].astype(np.float64)).reshape(rows, d)
        o = st.token_logprob(y @ hv, 1.0, target[mb])
        g = st.token_logprob_grad(o["all"], None, 1.0, target[mb], np.full(rows, -1.0 / (n_mb * rows)))
        assert so.max_rel_err(to_np(logp[mb]), o["logp"]) <= TOL[dtype]
        assert so.max_rel_err(to_np(dY[mb]), g @ hv.T) <= TOL[dtype]
        ref_dwh += y.T @ g
        dx = ref.backward_input(mb, (g @ hv.T).reshape(lay))
        assert so.max_rel_err(to_np(dX[mb]), dx.reshape(rows, d)) <= TOL[dtype]
        ref.backward_weight(mb)
    assert so.max_rel_err(to_np(dWh[:, :vocab]), ref_dwh) <= TOL[dtype]
    grads = stage.grads()
    for lg, lr in zip(grads, ref.grads):
        for k in lr:
            assert so.max_rel_err(lg[k], lr[k]) <= TOL[dtype], k
    # the norm over both, and the update
    total = torch.zeros(1, dtype=torch.float64, device="cuda:0")
    stage.grad_sumsq(total)
    scratch = torch.empty(L.stage_kernel_grad_sumsq_scratch_bytes(), dtype=torch.uint8, device="cuda:0")
    one = lambda *v: (C.c_void_p * len(v))(*v)
    assert L.stage_kernel_grad_sumsq(0, 1, (i64 * 1)(dWh.numel()), one(ptr(dWh)), 1, ptr(total), ptr(scratch), scratch.numel(), None) == 0
    sync()
    want = st.sumsq([lg[k] for lg in grads for k in lg] + [to_np(dWh)])
    assert abs(float(total) - want) <= 1e-12 * want
    norm, factor = math.sqrt(want), st.clip_factor(want, float(np.float32(0.3 * math.sqrt(want))))
    most = float(np.float32(0.3 * norm))
    state = stage.adamw_state()
    before = stage._weights.view(td).clone()
    hyper = dict(lr=0.01, beta1=0.9, beta2=0.95, eps=1e-4 * norm, weight_decay=0.1)
    stage.adamw(state, step=1, sumsq=total, max_norm=most, **hyper)
    sync()
    after, m, v = stage._weights.view(td), to_np(state["m"]), to_np(state["v"])
    x32 = to_np(state["master"]) if "master" in state else to_np(after)
    for name, off, size in stage.tensors():
        at = slice(off, off + size)
        g = to_np(stage.grads_tensor()[at]) * factor
        h = dict(hyper, weight_decay=0.1 if name[0] == "w" else 0.0)
        wx, wm, wv = st.adamw(to_np(before[at]), np.zeros(size), np.zeros(size), g, step=1, **h)
        assert np.abs(m[at] - wm).max() <= 8 * E * np.abs(g).max() and np.abs(v[at] - wv).max() <= 16 * E * (g * g).max()
        assert np.abs(x32[at] - wx).max() <= hyper["lr"] * 32 * E + 4 * E * np.abs(wx).max(), name
        if dtype == "bf16":
            assert (to_np(after[at]) == rnd(x32[at].astype(np.float32), "bf16")).all()
    # clip: the gradients themselves
    kept, got = stage.grads_tensor().clone(), torch.zeros(1, device="cuda:0")
    stage.clip_grads(total, most, got)
    sync()
    assert abs(float(got) - norm) <= 2 * E * norm
    assert np.abs(to_np(stage.grads_tensor()) - factor * to_np(kept)).max() <= 4 * E * factor * np.abs(to_np(kept)).max()
    # operands of another type, size or place are refused before anything is launched
    n = kept.numel()
    kept, weights = stage.grads_tensor().clone(), stage._weights.clone()
    short = {k: state[k][:n - 1] for k in state}
    for call in (lambda: stage.grad_sumsq(total.float()), lambda: stage.grad_sumsq(total.cpu()), lambda: stage.grad_sumsq(total[:0]),
                 lambda: stage.clip_grads(total.float(), most), lambda: stage.clip_grads(total, most, got.double()), lambda: stage.clip_grads(total, 0.0),
                 lambda: stage.adamw(short, step=1, **hyper), lambda: stage.adamw({k: state[k].double() for k in state}, step=1, **hyper),
                 lambda: stage.adamw(state, step=1, sumsq=total.float(), max_norm=most, **hyper), lambda: stage.adamw(state, step=0, **hyper),
                 lambda: stage.adamw({k: state[k].new_zeros(2 * n)[::2] for k in state}, step=1, **hyper)):
        with pytest.raises(S.StageError):
            call()
    sync()
    assert torch.equal(kept, stage.grads_tensor()) and torch.equal(weights, stage._weights)
    stage.zero_grads()
    stage.grad_sumsq(total)
    sync()
    assert float(total) == 0.0
    stage.close()


# ---------------------------------------------------------------------------
# graphs and streams
# ---------------------------------------------------------------------------
class Step:
    """All entries one behind the other, on buffers of its own"""

    def __init__(self, dtype, rows, vocab, top, sizes):
        import torch
        x, target, (w, dh, dl) = logits(rows, vocab, dtype, 77)
        self.one, self.two = Logprob(dtype, x, target, 1.3, top, w, dh, dl, (3, 3), (1, 1)), Logprob(dtype, x, target, 1.0, 0, w, None, None)
        self.up = Update(sizes, "bf16", "fp32", 1, 1)
        self.total, self.norm = torch.zeros(1, dtype=torch.float64, device="cuda:0"), torch.zeros(1, device="cuda:0")
        self.lr, self.step_now = torch.full((1,), 0.01, device="cuda:0"), torch.ones(1, dtype=torch.int32, device="cuda:0")
        self.clipped = List(sizes, [np.zeros(s, np.float32) for s in sizes], "fp32", 1, 1)
        self.scratch = torch.empty(self.one.L.stage_kernel_grad_sumsq_scratch_bytes(), dtype=torch.uint8, device="cuda:0")

    def load(self, seed):
        import torch
        g = torch.Generator(device="cuda:0").manual_seed(seed)
        for pr in (self.one, self.two):
            pr.x.copy_(torch.randn(pr.rows, pr.vocab, generator=g, device="cuda:0") * 2)
        self.step_now.fill_(seed)
        self.lr.fill_(0.001 * seed)
        self.up.lists["g"].buf.normal_(generator=g)
        for k, s in (("x", 1.0), ("m", 0.1)):
            self.up.lists[k].buf.normal_(generator=g).mul_(s)
        self.up.lists["v"].buf.normal_(generator=g).square_()

    def run(self, stream):
        L, g, c = self.one.L, self.up.lists["g"], self.clipped
        assert self.one.fwd(0, stream) == 0 and self.one.bwd(0, stream) == 0 and self.two.grad(0, stream, without=("entropy",)) == 0
        assert L.stage_kernel_grad_sumsq(0, g.n, g.c_sizes, g.ptrs, 0, ptr(self.total), ptr(self.scratch), self.scratch.numel(), stream) == 0
        assert L.stage_kernel_grad_clip(0, g.n, g.c_sizes, g.ptrs, c.ptrs, ptr(self.total), 2.0, ptr(self.norm), stream) == 0
        assert self.up.step(sumsq=self.total, max_norm=2.0, lr_now=self.lr, step_now=self.step_now, stream=stream) == 0

    def results(self):
        out = {f"{n}.{k}": v for n, pr in (("one", self.one), ("two", self.two)) for k, v in dict(pr.out, dx=pr.whole_dx).items() if not (n == "two" and k == "entropy")}
        out.update({k: l.buf for k, l in self.up.lists.items()}, clipped=self.clipped.buf, total=self.total, norm=self.norm)
        return {k: v.contiguous().view(-1).view(dtype=__import__("torch").uint8).clone() for k, v in out.items()}


STEPS = [("bf16", 5, 40000, 20, [1001, 7, 40000]), ("fp32", 300, 501, 5, [3] * 130), ("bf16", 1, 9000, 64, [70000])]


@pytest.mark.parametrize("dtype,rows,vocab,top,sizes", STEPS)
def test_captured_step(dtype, rows, vocab, top, sizes):
    """In a captured graph, replayed with new inputs, learning rates and step numbers, eager work in between: every replay the same bits as the eager calls."""
    import torch
    s = Step(dtype, rows, vocab, top, sizes)
    s.load(1)
    s.run(torch.cuda.current_stream().cuda_stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run(torch.cuda.current_stream().cuda_stream)
    for seed in (2, 3, 4, 5):
        s.load(seed)
        s.run(torch.cuda.current_stream().cuda_stream)
        sync()
        want = s.results()
        s.load(seed)
        for pr in (s.one, s.two):
            for v in pr.out.values():
                v.fill_(-5)
        junk = torch.randn(500, 500, device="cuda:0") @ torch.randn(500, 500, device="cuda:0")
        graph.replay()
        sync()
        assert bool(torch.isfinite(junk).all())
        for k, v in s.results().items():
            assert torch.equal(v, want[k]), (seed, k)


def test_two_streams():
    import torch
    a, b = Step(*STEPS[0]), Step(*STEPS[1])
    want = []
    for s, seed in ((a, 3), (b, 4)):
        s.load(seed)
        s.run(torch.cuda.current_stream().cuda_stream)
        sync()
        want.append(s.results())
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.load(3)
        b.load(4)
        sync()
        a.run(one.cuda_stream)
        b.run(two.cuda_stream)
        sync()
        for s, w in zip((a, b), want):
            for k, v in s.results().items():
                assert torch.equal(v, w[k]), k


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kernel_set", [0, 1, 2])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_two_million_rows(kernel_set, dtype):
    """The most rows there may be, against torch in 64 bits."""
    import torch
    rows, vocab = 1 << 21, 3
    x = np.random.default_rng(1).normal(0, 2, (rows, vocab)).astype(np.float32)
    pr = Logprob(dtype, rnd(x, dtype), np.arange(rows) % 5 - 1, 1.0, 2, np.ones(rows, np.float32))
    assert pr.fwd(kernel_set) == 0
    sync()
    y = torch.log_softmax(pr.x.double(), 1)
    t = pr.target.long()
    has = (t >= 0) & (t < vocab)
    want = torch.where(has, y.gather(1, t.clamp(0, vocab - 1)[:, None])[:, 0], 0.0)
    assert float((pr.out["logp"].double() - want).abs().max()) <= 64 * E
    best, where = torch.sort(pr.x.double(), dim=1, descending=True, stable=True)
    assert torch.equal(pr.out["top_id"].long(), where[:, :2])
    one_hot = torch.zeros_like(y).scatter_(1, t.clamp(0, vocab - 1)[:, None], has.double()[:, None])
    g = one_hot - y.exp() * has.double()[:, None]
    for both in (False, True):
        pr.dx.fill_(float("nan"))
        pr.p.top = 0
        assert (pr.grad(kernel_set) if both else pr.bwd(kernel_set)) == 0
        sync()
        assert float((pr.dx.double() - g).abs().max()) <= 64 * E + (2.0 ** -9 if dtype == "bf16" else 0)


@pytest.mark.parametrize("kernel_set", [0, 1, 2])
@pytest.mark.parametrize("dtype,vocab,top", [("bf16", 200001, 20), ("bf16", 1 << 22, 64), ("fp32", 131073, 5), ("fp32", 1 << 22, 0)])
def test_wide_vocabularies(kernel_set, dtype, vocab, top):
    """Beyond what a workgroup's registers hold, up to the widest, against torch in 64 bits."""
    import torch
    rows = 3
    x = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(vocab)).numpy() * 2
    pr = Logprob(dtype, rnd(x, dtype), [5, vocab - 1, -1], 1.0, top, np.ones(rows, np.float32), np.full(rows, 0.3, np.float32))
    assert pr.fwd(kernel_set) == 0 and pr.bwd(kernel_set) == 0
    sync()
    xd = pr.x.double().requires_grad_(True)
    y = torch.log_softmax(xd, 1)
    h = -(y.exp() * y).sum(1)
    want = torch.stack((y[0, 5], y[1, vocab - 1], torch.zeros_like(y[0, 0])))
    chain = (vocab / 256 + 64) * E
    assert float((pr.out["logp"].double() - want.detach()).abs().max()) <= chain
    assert float((pr.out["entropy"].double() - h.detach()).abs().max()) <= 16 * chain
    if top:
        best, where = torch.sort(pr.x.double(), dim=1, descending=True, stable=True)
        assert torch.equal(pr.out["top_id"].long(), where[:, :top])
        assert float((pr.out["top_logp"].double() - y.detach().gather(1, where[:, :top])).abs().max()) <= chain
    (g,) = torch.autograd.grad(want.sum() + 0.3 * h.sum(), xd)
    y, h = y.detach(), h.detach()
    bound = 64 * chain * y.exp() * (1 + 0.3 * (y.abs() + h[:, None])) + 2 * E + (2.0 ** -8 * g.abs() if dtype == "bf16" else 0)
    for both in (False, True):
        if both:
            pr.dx.fill_(float("nan"))
            assert pr.grad(kernel_set) == 0
            sync()
        assert bool(((pr.dx.double() - g).abs() <= bound).all())


@pytest.mark.parametrize("kernel_set", [0, 1, 2])
def test_rows_far_apart(kernel_set):
    """Row strides that pass 32 bits, of logits and gradient."""
    import torch
    ld, rows, vocab = (1 << 31) + 24, 3, 5003
    x, target, (w, dh, dl) = logits(rows, vocab, "bf16", 6)
    far = Logprob("bf16", x, target, 1.0, 5, w, dh, dl)
    near, buf = far.x, torch.empty((rows - 1) * ld + vocab + 64, dtype=torch.bfloat16, device="cuda:0")
    far.x = buf.as_strided((rows, vocab), (ld, 1), 8)
    far.x.copy_(near)
    assert far.fwd(kernel_set) == 0
    sync()
    ref = far.check_values()
    assert far.bwd(kernel_set, into=far.x) == 0
    sync()
    far.check_grad(ref, far.x)
    far.x.copy_(near)
    far.p.top = 0
    assert far.grad(kernel_set, into=far.x) == 0
    sync()
    far.check_grad(ref, far.x)


def test_a_tensor_of_four_thousand_million_elements():
    import torch
    from paper_2507_00217_amd import stage as S
    n = (1 << 32) + 77
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda:0")
    g[-1] = 4.0
    sizes, p = (C.c_int64 * 1)(n), (C.c_void_p * 1)(ptr(g))
    total, scratch = torch.zeros(1, dtype=torch.float64, device="cuda:0"), torch.empty(S.lib().stage_kernel_grad_sumsq_scratch_bytes(), dtype=torch.uint8, device="cuda:0")
    assert S.lib().stage_kernel_grad_sumsq(1, 1, sizes, p, 0, ptr(total), ptr(scratch), scratch.numel(), None) == 0
    sync()
    assert float(total) == (n - 1) * 0.25 + 16.0         # every partial sum is a multiple of a quarter below 2^51
    assert S.lib().stage_kernel_grad_clip(1, 1, sizes, p, p, ptr(total), 0.5 * math.sqrt(float(total)), None, None) == 0
    sync()
    assert float(g[-1]) == 2.0 and float(g[0]) == 0.25 and int((g == 0.25).sum()) == n - 1


def test_the_same_tensor_twice():
    """Gradients that two names share count twice in the norm of a list that names them twice."""
    v = values([100], 4)
    l = List([100], v, "fp32")
    l.t, l.sizes, l.n = l.t * 2, [100, 100], 2
    one = float((v[0].astype(np.float64) ** 2).sum())
    assert abs(float(sumsq("fp32", l)) - 2 * one) < 1e-12 * one


# ---------------------------------------------------------------------------
# which kernels the rules come to
# ---------------------------------------------------------------------------
def names_of(dtype, rows, vocab, top, mode, entropy):
    import torch
    from paper_2507_00217_amd import stage as S
    L, a = S.lib(), torch.zeros(64, device="cuda:0")
    q = ptr(a)
    p = S.TokenLogprob(dtype=DT[dtype], rows=rows, vocab=vocab, top=top, scale=1.0, target=q)
    h = q if entropy else None
    vals = [q, q, h, q, q, q, 1 << 60]
    call = {"score": lambda s: L.stage_kernel_token_logprob_fwd(C.byref(p), q, vocab, *vals, 0, s),
            "bwd": lambda s: L.stage_kernel_token_logprob_bwd(C.byref(p), q, vocab, q, q, q, h, None, q + 0, vocab, 0, s),
            "loss": lambda s: L.stage_kernel_token_logprob_grad(C.byref(p), q, vocab, q, h, None, q, vocab, *vals, 0, s)}[mode]
    return [n for n, _, _ in launches(call)]


def test_the_rules_reach_every_kernel():
    """Captured, never run."""
    found = set()
    for dtype, v in (("bf16", 8), ("fp32", 4)):
        for pieces in (10, 64, 65, 256, 300, 512, 600, 1024, 1500, 2048, 3000, 4096, 5000, 8192, 9000, 16384, 20000):
            for rows in (1, 100, 300, 1000, 5000, 1 << 19):
                for entropy in (False, True):
                    for top in (0, 5):
                        found.update(names_of(dtype, rows, pieces * v, top, "score", entropy))
                    found.update(names_of(dtype, rows, pieces * v, 0, "loss", entropy))
                    found.update(names_of(dtype, rows, pieces * v, 0, "bwd", entropy))
    short = {re.sub(r"^.*?(logprob\w*?_kernel)I(.*?)EEv.*$", r"\1 \2", n) for n in found}
    flag = ("Lb0E", "Lb1E")
    want = {f"logprob_kernel {t}Li{nt}E{a}{b}{c}" for t in ("DF16b", "f") for nt in (64, 256, 512) for a in flag for b in flag for c in flag}
    want |= {f"logprob_both_kernel {t}Li{nt}ELi{nv}ELi{nl}E{a}{b}" for t in ("DF16b", "f") for nt, nv, nl in ((64, 1, 0), (64, 4, 0), (64, 8, 4), (256, 4, 0), (256, 8, 4), (512, 8, 4), (512, 16, 8), (1024, 16, 8))
             for a in flag for b in flag}
    want |= {f"logprob_both_kernel {t}Li256ELi1ELi0E{a}Lb0E" for t in ("DF16b", "f") for a in flag}          # few rows of few columns: never large
    want |= {f"logprob_grad_kernel {t}{a}{b}" for t in ("DF16b", "f") for a in flag for b in flag}
    assert want == {n for n in short if "join" not in n}, sorted(want ^ short)
    assert any("logprob_join_kernel" in n for n in short)
