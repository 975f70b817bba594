"""Log probabilities and the logits' gradient on rows and sizes where kernels part: rows of nothing but NaN, ties below zero; and every form of the kernels
at sizes that come to it by themselves."""
import math

import numpy as np
import pytest

from tests.step_util import Logprob, logits

pytestmark = pytest.mark.gpu
SETS = [0, 1, 2]


def sync():
    import torch
    torch.cuda.synchronize()


def signalling(t, rows):
    """puts NaNs that are not quiet over the rows of a tensor"""
    import torch
    half = t.element_size() == 2
    t.view(torch.int16 if half else torch.int32)[rows] = 0x7f81 if half else 0x7f800001


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 9, 100, 700, 1500, 3500, 7001, 20003])
@pytest.mark.parametrize("top", [0, 3])
def test_rows_of_nan(kernel_set, dtype, vocab, top):
    """Nothing but NaN, NaN among -inf wherever it lies, signalling ones: the largest logit that is a number is -inf, as in a row without tokens, but such a row's gradient is zeros and these
    rows' is NaN, whose norm no update takes."""
    import torch
    from tests.test_gpu_grad_update import List, sumsq
    x, _, _ = logits(9, vocab, dtype, vocab)
    target, top = np.arange(9) % vocab, min(top, vocab)
    x[0] = x[5] = np.nan
    x[1:5] = -np.inf
    x[1, 0] = x[2, vocab // 2] = x[3, vocab - 1] = np.nan            # row 4: no token
    x[6, ::2] = np.nan
    x[6, 1::2] = -np.inf
    x[7, 0] = np.nan
    w, dh, dl = np.full(9, -0.5, np.float32), np.full(9, 0.25, np.float32), np.full(9, 0.125, np.float32)
    for grads in ((w, dh, dl), (w, None, None), (None, None, dl)):
        pr = Logprob(dtype, x, target, 1.0, top, *grads, (3, 3), (1, 1))
        signalling(pr.x, 5)
        assert pr.fwd(kernel_set) == 0 and pr.bwd(kernel_set) == 0
        sync()
        ref = pr.check_values()
        pr.check_grad(ref)
        first = pr.dx.clone()
        pr.dx.fill_(7.0)
        assert pr.grad(kernel_set) == 0
        sync()
        pr.check_values(ref)
        pr.check_grad(ref)
        for g in (first, pr.dx):
            assert bool(g[[0, 1, 2, 3, 5, 6, 7]].isnan().all()) and bool((g[4] == 0).all()) and bool(g[8].isfinite().all())
            one = List([vocab], [np.zeros(vocab)], dtype)
            for r in (0, 1, 3, 5):
                one.t[0].copy_(g[r])
                assert not math.isfinite(float(sumsq(dtype, one)))


def test_a_row_of_nan_in_a_share_of_the_vocabulary():
    """Statistics that a program has joined over shares: the share whose columns are all -inf has NaN where another share's logits made ln S NaN, zeros where no share has a token."""
    import torch
    for kernel_set in (0, 1):
        x = np.full((2, 300), -np.inf, np.float32)
        pr = Logprob("fp32", x, [-1, -1], 1.0, 0, None, None, [0.5, 0.5])
        pr.out["stats"].copy_(torch.tensor([[-math.inf, math.nan], [-math.inf, -math.inf]]))
        assert pr.bwd(kernel_set) == 0
        sync()
        assert bool(pr.dx[0].isnan().all()) and bool((pr.dx[1] == 0).all())


def tied(how, vocab, dtype):
    """One row whose alternatives are decided among equal logits"""
    import torch
    from tests.gpu_util import rnd
    rng, low = np.random.default_rng(3), float(torch.finfo(torch.float32 if dtype == "fp32" else torch.bfloat16).min)
    left = np.isin(np.arange(vocab), rng.integers(0, vocab, 9))
    kinds = {"constant": np.full(vocab, -1.0), "small": np.full(vocab, -1e-30), "two values": np.where(rng.random(vocab) < 0.5, -1.0, -2.0), "lowest": np.full(vocab, low),
             "few left": np.where(left, rng.normal(0, 1, vocab), -1e4), "few left, lowest": np.where(left, rng.normal(0, 1, vocab), low),
             "few left, negative": np.where(left, rng.normal(-9, 1, vocab), -1e4), "above": np.full(vocab, 1.0), "zero": np.zeros(vocab)}
    return rnd(kinds[how], dtype)


TIES = ["constant", "small", "two values", "lowest", "few left", "few left, lowest", "few left, negative"]


@pytest.mark.parametrize("kernel_set", SETS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,top", [(700, 40), (3300, 64), (5000, 64), (40000, 20)])
@pytest.mark.parametrize("how", TIES)
def test_ties_below_zero(kernel_set, dtype, vocab, top, how):
    x = tied(how, vocab, dtype)
    pr = Logprob(dtype, np.stack((x, x)), [1, vocab - 1], 1.0, top)
    assert pr.fwd(kernel_set) == 0
    sync()
    pr.check_values()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("how", TIES)
def test_what_ties_take(dtype, how):
    """The way made for ties finds them in one more pass over a row: twice what rows of zeros take is room for another share of rows that take it (or the walk a second time, which the lowest values make).
    One by one, `top` passes, was 8 times and more."""
    import torch
    from tests.test_gpu_score_odd import once
    rows, vocab, top = 512, 40000, 40
    time = {}
    for kind in ("zero", how):
        pr = Logprob(dtype, np.broadcast_to(tied(kind, vocab, dtype), (rows, vocab)), None, 1.0, top)
        stream = torch.cuda.current_stream().cuda_stream
        time[kind] = once(lambda: pr.fwd(0, stream))
    assert time[how] <= 2 * time["zero"], time


# ---------------------------------------------------------------------------
# values and gradient in one call, in every form of the kernel that holds rows in registers
# ---------------------------------------------------------------------------
# threads of a workgroup, pieces of 16 bytes to each, rows, columns in bf16 (half as many in fp32).  Rows are more than the workgroups that are launched, but where the form is for few rows.
FORMS = {"64x1": (64, 1, 8500, 333), "256x1": (256, 1, 300, 1501), "64x4": (64, 4, 8300, 1203), "64x8": (64, 8, 6200, 3001), "256x4": (256, 4, 2100, 6001), "256x8": (256, 8, 1600, 9001),
         "512x8": (512, 8, 800, 17001), "512x16": (512, 16, 700, 40001), "1024x16": (1024, 16, 300, 70001),
         # the widest rows, and more logits and gradient than the caches are asked to keep
         "1024x16 full": (1024, 16, 515, 131072), "512x8 large": (512, 8, 2200, 32003)}


class OneCall:
    """Logits made on the GPU, an offset and a spread of their own to each row; some rows are odd.  ld: columns from one row to the next; dx_shift: where the gradient's buffer starts."""

    def __init__(self, dtype, rows, vocab, pad=0, shift=0, dx_pad=0, dx_shift=0, in_place=False, entropy=True, odd=True, scale=0.8, seed=0, top=0):
        import ctypes as C

        import torch
        from paper_2507_00217_amd import stage as S
        from tests.score_util import DT
        self.C, self.S, td = C, S, torch.float32 if dtype == "fp32" else torch.bfloat16
        g = torch.Generator(device="cuda:0").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda:0")
        self.buf = torch.full((rows, shift + vocab + pad), math.nan, dtype=td, device="cuda:0")
        self.x = self.buf[:, shift:shift + vocab]
        std = torch.rand(rows, 1, generator=g, device="cuda:0") * 4.0 + 0.5
        self.x.copy_(normal(rows, vocab).mul_(std).add_(normal(rows, 1) * 4.0))
        self.target = torch.randint(-1, vocab, (rows,), generator=g, device="cuda:0", dtype=torch.int32)
        self.w, self.dh, self.dl = normal(rows), normal(rows) if entropy else None, normal(rows)
        if odd:                                        # early rows, and late ones, which a workgroup comes to behind others
            last = vocab - 1
            for base in (3, rows - 13):
                self.x[base] = math.nan
                self.x[base + 1] = -math.inf
                self.x[base + 2, last] = math.inf
                self.x[base + 3, vocab // 2] = math.nan
                self.x[base + 4, 1:] = -math.inf
                self.x[base + 4, 0] = 2.0
                self.x[base + 5, ::2] = -math.inf
                self.x[base + 6] = -1.5
                self.x[base + 7, vocab // 3] = 200.0         # certain
                self.target[base:base + 8] = torch.tensor([0, last, 1, 2, 0, 1, last, vocab // 3], dtype=torch.int32)
                for v in (self.w, self.dh, self.dl):
                    if v is not None:
                        v[base + 8] = v[base + 9] = 0.0      # zeros, whatever the logits are
                self.x[base + 9] = math.nan
        self.kept = self.x.clone()
        if in_place:
            self.dbuf, self.dx = self.buf, self.x
        else:
            self.dbuf = torch.full((rows, dx_shift + vocab + dx_pad), math.nan, dtype=td, device="cuda:0")
            self.dx = self.dbuf[:, dx_shift:dx_shift + vocab]
            self.dx.fill_(7.0)
        self.outside = torch.ones(self.dbuf.shape[1], dtype=torch.bool, device="cuda:0")
        self.outside[self.dx.storage_offset():self.dx.storage_offset() + vocab] = False
        self.scale, self.rows, self.vocab = scale, rows, vocab
        self.p = S.TokenLogprob(dtype=DT[dtype], rows=rows, vocab=vocab, top=top, scale=scale, target=self.target.data_ptr())
        self.out = dict(logp=torch.full((rows,), -9.0, device="cuda:0"), stats=torch.full((rows, 2), -9.0, device="cuda:0"))
        if entropy:
            self.out["entropy"] = torch.full((rows,), -9.0, device="cuda:0")
        if top:
            self.out.update(top_id=torch.full((rows, top), -7, dtype=torch.int32, device="cuda:0"), top_logp=torch.full((rows, top), -9.0, device="cuda:0"))
        self.scratch = torch.empty(S.lib().stage_kernel_token_logprob_scratch_bytes(C.byref(self.p)) + 16, dtype=torch.uint8, device="cuda:0")

    def values(self):
        ptr = lambda t: None if t is None else t.data_ptr()
        return [ptr(self.out.get(k)) for k in ("logp", "stats", "entropy", "top_id", "top_logp")] + [ptr(self.scratch), self.scratch.numel()]

    def fwd(self, stream, kernel_set=0):
        return self.S.lib().stage_kernel_token_logprob_fwd(self.C.byref(self.p), self.x.data_ptr(), self.x.stride(0), *self.values(), kernel_set, stream)

    def grad(self, stream, kernel_set=0):
        return self.S.lib().stage_kernel_token_logprob_grad(self.C.byref(self.p), self.x.data_ptr(), self.x.stride(0), *(None if v is None else v.data_ptr() for v in (self.w, self.dh, self.dl)),
                                                            self.dx.data_ptr(), self.dx.stride(0), *self.values(), kernel_set, stream)

    def check(self, chain, grad=True):
        from tests.step_exact import Rows
        rows, block = self.rows, max(1, (1 << 25) // self.vocab)
        for i in range(0, rows, block):
            at = slice(i, min(rows, i + block))
            ref = Rows(self.kept[at], self.scale, self.target[at], chain)
            ref.check_values(**{k: self.out[k][at] for k in ("logp", "stats", "entropy") if k in self.out})
            if grad:
                ref.check_grad(self.dx[at], *(None if v is None else v[at] for v in (self.w, self.dh, self.dl)))
        if grad:
            assert bool(self.dbuf[:, self.outside].isnan().all())


LAYOUTS = {"dense": {}, "odd, apart": dict(pad=3, shift=1, dx_pad=2, dx_shift=2), "odd, alike": dict(pad=2, shift=3, dx_pad=2, dx_shift=3), "in place": dict(pad=1, shift=1, in_place=True)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_one_call_in_every_form(form, dtype, entropy, layout):
    """Every form holds the row that it is made for, goes on to next rows whose first pieces lie elsewhere, and stores the gradient in whole pieces, element by element and over the logits; rows that
    are not finite, that have no token and that have no weights are among the first and the last ones.  Additions behind one another: a thread's elements and two edges, 12 of lanes and wavefronts."""
    import re

    import torch
    from tests.gpu_util import launches
    threads, pieces, rows, vocab = FORMS[form]
    if dtype == "fp32":
        vocab = (vocab + 1) // 2
    q = OneCall(dtype, rows, vocab, entropy=entropy, seed=len(form) + vocab, **LAYOUTS[layout])
    ((name, groups, _),) = launches(q.grad)
    assert re.search(rf"logprob_both_kernelI(DF16b|f)Li{threads}ELi{pieces}ELi\d+ELb{int(entropy)}ELb{int('large' in form or 'full' in form)}E", name), name
    assert groups < rows or pieces == 1 and rows <= 512, (groups, rows)
    assert q.grad(torch.cuda.current_stream().cuda_stream) == 0
    sync()
    q.check(pieces * (4 if dtype == "fp32" else 8) + 14)


@pytest.mark.parametrize("form", ["64x8", "256x8", "512x8", "512x16", "1024x16"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_two_calls_at_once_and_again(form, dtype):
    """The forms that bring the next row to LDS: two problems on two streams, over the logits too, and replayed from a graph, always the same bits."""
    import torch
    _, _, rows, vocab = FORMS[form]
    both = [OneCall(dtype, rows, vocab, in_place=i == 1, pad=1, shift=1, entropy=i == 0, seed=i) for i in (0, 1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    want = None
    bits = lambda q: [v.contiguous().view(torch.uint8).clone() for v in (q.dx, *q.out.values())]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for q in both:
            assert q.grad(torch.cuda.current_stream().cuda_stream) == 0
    for turn in range(6):
        for q in both:
            q.x.copy_(q.kept)
            for v in q.out.values():
                v.fill_(-5.0)
        sync()
        if turn % 2 == 0:
            for q, s in zip(both, streams):
                assert q.grad(s.cuda_stream) == 0
        else:
            graph.replay()
        sync()
        got = [bits(q) for q in both]
        want = want or got
        for a, b in zip(want, got):
            assert all(torch.equal(u, v) for u, v in zip(a, b)), turn


# rows beyond what registers hold, and few wide ones; additions behind one another: a thread's elements, six roundings for each group of two pieces that the walk comes to, 28 of edges, lanes,
# wavefronts and parts
WIDE = [("bf16", 300, 140001, 35 * 8 + 18 * 6 + 28), ("fp32", 300, 70001, 35 * 4 + 18 * 6 + 28), ("bf16", 40, 200001, 3 * 8 + 2 * 6 + 28), ("fp32", 40, 131073, 3 * 8 + 2 * 6 + 28),
        ("bf16", 20, 1 << 22, 32 * 8 + 16 * 6 + 28), ("fp32", 20, 1 << 22, 64 * 4 + 32 * 6 + 28)]


@pytest.mark.parametrize("kernel_set", [0, 2])
@pytest.mark.parametrize("dtype,rows,vocab,chain", WIDE)
@pytest.mark.parametrize("layout", ["dense", "odd, apart", "in place"])
def test_one_call_of_wide_rows(kernel_set, dtype, rows, vocab, chain, layout):
    """In three launches: the walk (in parts, joined), then the gradient from its statistics."""
    import torch
    q = OneCall(dtype, rows, vocab, seed=vocab, **LAYOUTS[layout])
    assert q.grad(torch.cuda.current_stream().cuda_stream, kernel_set) == 0
    sync()
    q.check(chain)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("rows,vocab,threads", [(21000, 6500, 256), (17000, 8500, 256), (65000, 2200, 64), (1100, 131071, 512)])
@pytest.mark.parametrize("top", [0, 20])
def test_values_of_more_logits_than_the_caches_keep(dtype, entropy, rows, vocab, threads, top):
    """The walk's form for more than 256 MB of logits, with alternatives and without; a part of the rows' alternatives against a stable sort."""
    import re

    import torch
    from tests.gpu_util import launches
    if dtype == "fp32":
        vocab = (vocab + 1) // 2
    if vocab * (2 if dtype == "fp32" else 1) <= 8192 and top == 0:      # without alternatives one wavefront goes further
        threads = 64
    q = OneCall(dtype, rows, vocab, pad=1, shift=1, entropy=entropy, seed=rows + top, top=top, in_place=True)
    ((name, _, _),) = launches(q.fwd)
    assert re.search(rf"14logprob_kernelI(DF16b|f)Li{threads}ELb{int(top > 0)}ELb{int(entropy)}ELb1E", name), name
    assert q.fwd(torch.cuda.current_stream().cuda_stream) == 0
    sync()
    each = -(-vocab // (threads * (4 if dtype == "fp32" else 8)))
    q.check((each + 1) * (4 if dtype == "fp32" else 8) + (each // 2 + 1) * 6 + 28, grad=False)
    if top:
        from tests.step_exact import E
        some = torch.cat((torch.arange(0, 40), torch.arange(40, rows - 40, rows // 40), torch.arange(rows - 40, rows))).to("cuda:0")
        x, ids, lp = q.x[some].float(), q.out["top_id"][some].long(), q.out["top_logp"][some]
        bad = (x.isnan() | (x == math.inf)).any(1)
        assert bool((ids[bad] == -1).all()) and bool(lp[bad].isnan().all()) and int(bad.sum()) >= 6
        best, where = torch.sort(x[~bad], dim=1, descending=True, stable=True)
        assert torch.equal(ids[~bad], where[:, :top])
        # z - ln S from the kernel's own ln S, which is checked above: three roundings of z, one of the difference
        m, ln = (q.out["stats"][some][~bad][:, i:i + 1].double() for i in (0, 1))
        z = float(np.float32(q.scale)) * (best[:, :top].double() - torch.where(m == -math.inf, 0.0, m))
        want = torch.where(z == -math.inf, z, z - ln)
        got = lp[~bad].double()
        same = (got == want) | ((got - want).abs() <= 3 * E * z.abs() + E * want.abs())
        assert bool(same.all()), (got[~same][:4], want[~same][:4])
