"""Log probabilities and the logits' gradient on rows and sizes where kernels part: rows of nothing but NaN, ties below zero."""
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

    def __init__(self, dtype, rows, vocab, pad=0, shift=0, dx_pad=0, dx_shift=0, in_place=False, entropy=True, odd=True, scale=0.8, seed=0):
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
        self.p = S.TokenLogprob(dtype=DT[dtype], rows=rows, vocab=vocab, top=0, scale=scale, target=self.target.data_ptr())
        self.out = dict(logp=torch.full((rows,), -9.0, device="cuda:0"), stats=torch.full((rows, 2), -9.0, device="cuda:0"))
        if entropy:
            self.out["entropy"] = torch.full((rows,), -9.0, device="cuda:0")
        self.scratch = torch.empty(S.lib().stage_kernel_token_logprob_scratch_bytes(C.byref(self.p)) + 16, dtype=torch.uint8, device="cuda:0")

    def grad(self, stream):
        ptr = lambda t: None if t is None else t.data_ptr()
        o = self.out
        return self.S.lib().stage_kernel_token_logprob_grad(self.C.byref(self.p), ptr(self.x), self.x.stride(0), ptr(self.w), ptr(self.dh), ptr(self.dl), ptr(self.dx), self.dx.stride(0), ptr(o["logp"]),
                                                            ptr(o["stats"]), ptr(o.get("entropy")), None, None, ptr(self.scratch), self.scratch.numel(), 0, stream)

    def check(self, chain):
        from tests.step_exact import Rows
        rows, block = self.rows, max(1, (1 << 25) // self.vocab)
        for i in range(0, rows, block):
            at = slice(i, min(rows, i + block))
            ref = Rows(self.kept[at], self.scale, self.target[at], chain)
            ref.check_values(**{k: v[at] for k, v in self.out.items()})
            ref.check_grad(self.dx[at], *(None if v is None else v[at] for v in (self.w, self.dh, self.dl)))
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
