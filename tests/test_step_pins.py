"""Pins of oracle/step_oracle.py (differences, torch autograd, torch.optim, hand values) and what the library's entries around a training step refuse.
Runs without a GPU: refused calls launch nothing."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import step_oracle as st


def inputs(rows=5, vocab=9, seed=0):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 3, (rows, vocab))
    x[1, 3] = -np.inf
    target = rng.integers(0, vocab, rows)
    target[1], target[2], target[4] = 5, -1, vocab
    return x, target, [rng.normal(0, 1, rows) for _ in range(3)]


@pytest.mark.parametrize("scale", [1.0, 0.6, 2.5])
def test_logprob_against_torch(scale):
    import torch
    x, target, _ = inputs()
    o = st.token_logprob(x, scale, target, 4)
    y = torch.log_softmax(torch.tensor(x) * scale, 1)
    has = (target >= 0) & (target < x.shape[1])
    want = np.where(has, y.numpy()[np.arange(5), np.where(has, target, 0)], 0.0)
    assert np.allclose(o["logp"], want, atol=1e-13, rtol=0)
    assert np.allclose(o["stats"][:, 0], x.max(1)) and np.allclose(scale * o["stats"][:, 0] + o["stats"][:, 1], torch.logsumexp(torch.tensor(x) * scale, 1), atol=1e-13)
    assert np.allclose(o["entropy"], torch.special.entr(torch.softmax(torch.tensor(x) * scale, 1)).sum(1), atol=1e-13)
    assert np.allclose(o["top_logp"], torch.topk(y, 4).values, atol=1e-13) and (o["top_id"] == torch.topk(y, 4).indices.numpy()).all()


@pytest.mark.parametrize("scale", [1.0, 0.6])
def test_logprob_gradient_by_differences(scale):
    x, target, (w, dh, dl) = inputs()

    def f(v):
        o = st.token_logprob(v, scale, target)
        return (w * o["logp"] + dh * o["entropy"] + dl * (scale * o["stats"][:, 0] + o["stats"][:, 1])).sum()
    o = st.token_logprob(x, scale, target)
    g = st.token_logprob_grad(o["all"], o["entropy"], scale, target, w, dh, dl)
    assert g[1, 3] == 0.0
    for r in range(5):
        for j in range(9):
            if np.isfinite(x[r, j]):
                a, b = x.copy(), x.copy()
                a[r, j] += 1e-5
                b[r, j] -= 1e-5
                assert abs((f(a) - f(b)) / 2e-5 - g[r, j]) < 1e-8


def test_logprob_of_rows_at_the_edge():
    inf, nan = np.inf, np.nan
    x = np.array([[-inf, -inf, -inf], [2.0, 2.0, 2.0], [0.0, inf, 1.0], [0.0, nan, 1.0], [-3e38, -3e38, -3e38], [-inf, 7.0, -inf], [0.0, -0.0, 1.0]])
    o = st.token_logprob(x, 1.0, [0, 1, 2, 2, 0, 1, 0], 3)
    third = math.log(1 / 3)
    assert o["logp"][0] == -inf and o["entropy"][0] == 0.0 and list(o["top_id"][0]) == [0, 1, 2]
    assert abs(o["logp"][1] - third) < 1e-15 and abs(o["entropy"][1] + third) < 1e-15 and list(o["top_id"][1]) == [0, 1, 2]
    assert np.isnan(o["logp"][2:4]).all() and np.isnan(o["entropy"][2:4]).all() and (o["top_id"][2:4] == -1).all()
    assert abs(o["logp"][4] - third) < 1e-15
    assert o["logp"][5] == 0.0 and o["entropy"][5] == 0.0 and list(o["top_id"][5]) == [1, 0, 2] and list(o["top_logp"][5]) == [0.0, -inf, -inf]
    assert list(o["top_id"][6]) == [2, 0, 1]
    g = st.token_logprob_grad(o["all"], o["entropy"], 1.0, [0, 1, 2, 2, 0, 1, 0], np.ones(7), empty=o["stats"][:, 0] == -inf)
    assert (g[0] == 0).all() and np.allclose(g[1], [-1 / 3, 2 / 3, -1 / 3]) and np.isnan(g[2:4]).all() and (g[5] == 0).all()


def test_a_share_of_the_vocabulary_has_its_share_of_the_gradient():
    """Where a row's token lies on another share, its weight is a part of the row's dlse."""
    x, target, (w, dh, dl) = inputs()
    o = st.token_logprob(x, 0.7, target)
    whole = st.token_logprob_grad(o["all"], o["entropy"], 0.7, target, w, dh, dl)
    for first, cols in ((0, slice(0, 4)), (4, slice(4, 9))):
        here = target - first
        elsewhere = (target >= 0) & (target < 9) & ((here < 0) | (here >= cols.stop - first))
        part = st.token_logprob_grad(o["all"][:, cols], o["entropy"], 0.7, here, w, dh, dl - np.where(elsewhere, w, 0.0))
        assert np.allclose(part, whole[:, cols], atol=1e-14)


def test_clip_and_adamw_against_torch():
    import torch
    rng = np.random.default_rng(3)
    ws, gs = [rng.normal(0, 1, s) for s in ((7,), (3, 5))], [rng.normal(0, 2, s) for s in ((7,), (3, 5))]
    params = [torch.nn.Parameter(torch.tensor(w)) for w in ws]
    opt = torch.optim.AdamW(params, lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    m, v = [np.zeros_like(w) for w in ws], [np.zeros_like(w) for w in ws]
    for step in (1, 2, 3):
        for p, g in zip(params, gs):
            p.grad = torch.tensor(g * step)
        total = st.sumsq([g * step for g in gs])
        norm = torch.nn.utils.clip_grad_norm_(params, 1.5)
        assert abs(math.sqrt(total) - float(norm)) < 1e-12
        f = st.clip_factor(total, 1.5)
        opt.step()
        for i in range(2):
            ws[i], m[i], v[i] = st.adamw(ws[i], m[i], v[i], f * step * gs[i], 0.01, 0.8, 0.95, 1e-6, 0.1, step)
            assert np.allclose(ws[i], params[i].detach().numpy(), atol=1e-7)      # torch adds 1e-6 to the norm
    assert st.clip_factor(4.0, 2.0) == 1.0 and st.clip_factor(0.0, 1.0) == 1.0 and st.clip_factor(16.0, 1.0) == 0.25
    assert st.clip_factor(math.inf, 1.0) == 1.0 and st.clip_factor(math.nan, 1.0) == 1.0


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
def A(off=0):
    return 0x10000 + off


def tlp(**kw):
    from paper_2507_00217_amd import stage as S
    return S.TokenLogprob(**dict(dict(dtype=1, rows=4, vocab=100, top=0, scale=0.0, target=A()), **kw))


BIG = 1 << 40


def fwd(p, x=A(), ld=100, logp=A(), stats=A(), entropy=A(), ids=A(), tops=A(), scratch=A(), n=BIG):
    from paper_2507_00217_amd import stage as S
    return S.lib().stage_kernel_token_logprob_fwd(p, x, ld, logp, stats, entropy, ids, tops, scratch, n, 0, None)


def bwd(p, x=A(), ld=100, stats=A(), entropy=A(), w=A(), dh=A(), dl=A(), dx=A(1 << 20), ldd=100):
    from paper_2507_00217_amd import stage as S
    return S.lib().stage_kernel_token_logprob_bwd(p, x, ld, stats, entropy, w, dh, dl, dx, ldd, 0, None)


def grad(p, x=A(), ld=100, w=A(), dh=A(), dl=A(), dx=A(1 << 20), ldd=100, logp=A(), stats=A(), entropy=A(), ids=A(), tops=A(), scratch=A(), n=BIG):
    from paper_2507_00217_amd import stage as S
    return S.lib().stage_kernel_token_logprob_grad(p, x, ld, w, dh, dl, dx, ldd, logp, stats, entropy, ids, tops, scratch, n, 0, None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dtype=-1), dict(rows=0), dict(rows=-1), dict(rows=(1 << 21) + 1), dict(vocab=0), dict(vocab=(1 << 22) + 1), dict(top=-1),
                                dict(top=65), dict(vocab=10, top=11), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-31), dict(scale=1e31),
                                dict(target=A(2))])
def test_logprob_refuses_the_problem(kw):
    from paper_2507_00217_amd import stage as S
    p = C.byref(tlp(**kw))
    for f in (fwd, bwd, grad):
        assert f(p, ld=1 << 25, **({"ldd": 1 << 25} if f is not fwd else {})) == S.E_INVAL
        assert f(None) == S.E_INVAL
    assert S.lib().stage_kernel_token_logprob_scratch_bytes(p) == 0


def test_logprob_refuses_the_tensors():
    from paper_2507_00217_amd import stage as S
    p, wide, top, free = (C.byref(tlp(**k)) for k in ({}, dict(dtype=0), dict(top=5), dict(target=None)))
    for f in (fwd, bwd, grad):
        assert f(p, x=None) == S.E_INVAL and f(p, ld=99) == S.E_INVAL and f(p, x=A(1)) == S.E_INVAL and f(wide, x=A(2)) == S.E_INVAL
    for f in (fwd, grad):
        assert f(top, ids=None) == S.E_INVAL and f(top, tops=None) == S.E_INVAL
    for f in (bwd, grad):
        assert f(p, dx=None) == S.E_INVAL and f(p, ldd=99) == S.E_INVAL and f(p, dx=A(1)) == S.E_INVAL and f(p, dx=A(), ldd=101) == S.E_INVAL
        assert f(p, stats=None) == S.E_INVAL and f(p, entropy=None) == S.E_INVAL and f(p, w=None, dh=None, dl=None) == S.E_INVAL
        assert f(free) == S.E_INVAL


def test_logprob_refuses_the_scratch():
    from paper_2507_00217_amd import stage as S
    for kw in (dict(rows=1, vocab=200000), dict(rows=1, vocab=200000, top=64, dtype=0), dict(rows=3, vocab=1 << 22)):
        p = tlp(**kw)
        n = S.lib().stage_kernel_token_logprob_scratch_bytes(C.byref(p))
        assert n > 0
        for f in (fwd, grad):
            more = {} if f is fwd else dict(ldd=p.vocab)
            assert f(C.byref(p), ld=p.vocab, scratch=None, **more) == S.E_INVAL and f(C.byref(p), ld=p.vocab, n=n - 1, **more) == S.E_INVAL
            assert f(C.byref(p), ld=p.vocab, scratch=A(8), **more) == S.E_INVAL


def ptrs(*v):
    return (C.c_void_p * max(1, len(v)))(*v)


def sizes(*v):
    return (C.c_int64 * max(1, len(v)))(*v)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(n=-1), dict(size=None), dict(size=sizes(8, -1)), dict(size=sizes(8, BIG + 1)), dict(grad=None),
                                dict(grad=ptrs(A(), None)), dict(grad=ptrs(A(2), A())), dict(add=2), dict(total=None), dict(total=A(4)), dict(scratch=None),
                                dict(scratch=A(8)), dict(n_scratch=1)])
def test_sumsq_refuses(kw):
    from paper_2507_00217_amd import stage as S
    a = dict(dict(dtype=0, n=2, size=sizes(8, 8), grad=ptrs(A(), A()), add=0, total=A(), scratch=A(), n_scratch=BIG), **kw)
    assert S.lib().stage_kernel_grad_sumsq(a["dtype"], a["n"], a["size"], a["grad"], a["add"], a["total"], a["scratch"], a["n_scratch"], None) == S.E_INVAL


@pytest.mark.parametrize("kw", [dict(dtype=-1), dict(n=-1), dict(size=None), dict(size=sizes(8, -1)), dict(grad=None), dict(grad=ptrs(A(), None)), dict(out=None), dict(out=ptrs(None, A())),
                                dict(out=ptrs(A(1), A())), dict(total=None), dict(total=A(4)), dict(most=0.0), dict(most=-1.0), dict(most=math.inf), dict(most=math.nan),
                                dict(norm=A(2))])
def test_clip_refuses(kw):
    from paper_2507_00217_amd import stage as S
    a = dict(dict(dtype=1, n=2, size=sizes(8, 8), grad=ptrs(A(), A()), out=ptrs(A(), A()), total=A(), most=1.0, norm=A()), **kw)
    assert S.lib().stage_kernel_grad_clip(a["dtype"], a["n"], a["size"], a["grad"], a["out"], a["total"], a["most"], a["norm"], None) == S.E_INVAL


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(grad_dtype=3), dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.inf),
                                dict(eps=-1.0), dict(weight_decay=math.inf), dict(step=0), dict(sumsq=A(4)), dict(sumsq=A(), max_norm=0.0), dict(sumsq=A(), max_norm=math.inf),
                                dict(lr_now=A(1)), dict(step_now=A(2)), dict(n=-1), dict(size=sizes(-1)), dict(w=None), dict(w=ptrs(None)), dict(w=ptrs(A(1))), dict(master=None),
                                dict(master=ptrs(None)), dict(m=ptrs(A(2))), dict(v=None), dict(grad=ptrs(A(2))), dict(dtype=0)])
def test_adamw_refuses(kw):
    from paper_2507_00217_amd import stage as S
    kw = dict(kw)
    lists = dict(n=1, size=sizes(8), w=ptrs(A()), master=ptrs(A()), m=ptrs(A()), v=ptrs(A()), grad=ptrs(A()))
    lists.update({k: kw.pop(k) for k in list(kw) if k in lists})
    p = S.AdamW(**dict(dict(dtype=1, grad_dtype=0, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1), **kw))
    assert S.lib().stage_kernel_adamw(C.byref(p), *lists.values(), None) == S.E_INVAL
    assert S.lib().stage_kernel_adamw(None, *lists.values(), None) == S.E_INVAL
