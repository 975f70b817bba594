"""Pins of oracle/score_oracle.py (differences, closed forms, plain causal attention) and what the entries refuse.  Runs without a GPU:
refused calls launch nothing."""
import ctypes as C

import numpy as np
import pytest

from oracle import score_oracle as sc


def normal(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


OPTIONS = dict(plain={}, cap=dict(cap=2.0), bias=dict(slopes=[0.5, 0.0625]), packed=dict(starts=[1, 4, 4, 9], n_seq=3, prefixes=[2, 0, 9]),
               every=dict(cap=1.5, slopes=[0.3, -0.1], starts=[0, 7, 11], n_seq=2, prefixes=[3, 0], scale=0.7))


@pytest.mark.parametrize("name", list(OPTIONS))
@pytest.mark.parametrize("causal", [1, 0])
def test_attention_backward_against_differences(name, causal):
    opts = dict(OPTIONS[name], h=2, hkv=1, causal=causal)
    if not causal:
        opts["prefixes"] = None
    rows, hd = 11, 4
    t = dict(q=normal(1, rows, 2 * hd), k=normal(2, rows, hd), v=normal(3, rows, hd))
    do = normal(4, rows, 2 * hd)
    loss = lambda: float(np.nansum(sc.attention(**t, **opts)[0] * do))
    o, lse, _ = sc.attention(**t, **opts)
    grads = sc.attention_backward(**t, o=np.nan_to_num(o), lse=np.nan_to_num(lse), do=do, **opts)
    rng = np.random.default_rng(5)
    for n in "qkv":
        g = np.nan_to_num(grads["d" + n][0])
        for _ in range(12):
            i = tuple(rng.integers(0, s) for s in t[n].shape)
            was, e = t[n][i], 1e-5
            t[n][i] = was + e
            up = loss()
            t[n][i] = was - e
            down = loss()
            t[n][i] = was
            assert abs((up - down) / (2 * e) - g[i]) <= 1e-7 * (1.0 + abs(g[i])), (n, i)


def test_plain_options_are_the_engines_attention():
    """One sequence, no cap, no bias: the attention of the stage's oracle."""
    s, h, hkv, hd = 13, 4, 2, 8
    q, k, v = normal(6, s, h * hd), normal(7, s, hkv * hd), normal(8, s, hkv * hd)
    o, lse, _ = sc.attention(q, k, v, h, hkv, 1)
    for j in range(h):
        a = q[:, j * hd:(j + 1) * hd] @ k[:, j // 2 * hd:(j // 2 + 1) * hd].T / np.sqrt(hd)
        a = np.where(np.tril(np.ones((s, s), bool)), a, -np.inf)
        p = np.exp(a - a.max(1, keepdims=True))
        assert np.allclose(o[:, j * hd:(j + 1) * hd], p / p.sum(1, keepdims=True) @ v[:, j // 2 * hd:(j // 2 + 1) * hd], rtol=0, atol=1e-12)
        assert np.allclose(lse[j], np.log(np.exp(a).sum(1)), rtol=0, atol=1e-12)


def test_packing_is_separate_calls_and_prefix_opens_the_mask():
    rows, hd = 12, 4
    q, k, v = (normal(i, rows, hd) for i in (9, 10, 11))
    o, lse, _ = sc.attention(q, k, v, 1, 1, 1, starts=[2, 5, 11], n_seq=2, prefixes=[0, 4])
    a, la, _ = sc.attention(q[2:5], k[2:5], v[2:5], 1, 1, 1)
    assert np.array_equal(o[2:5], a) and np.array_equal(lse[:, 2:5], la)
    assert np.isnan(o[:2]).all() and np.isnan(o[11:]).all()
    full, _, _ = sc.attention(q[5:9], k[5:9], v[5:9], 1, 1, 0)
    assert np.allclose(o[5:9], full, rtol=0, atol=1e-14)                # the prefix sees all of itself, and nothing behind


@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("section,restart", [([4], 0), ([1, 3], 0), ([2, 1, 1], 1)])
def test_rotation(halves, section, restart):
    """Lengths stay, the way back undoes it, products of rotated heads depend on differences of positions only."""
    hd, rows = 8, 9
    pos = np.random.default_rng(1).integers(0, 50, (len(section), rows))
    x, y = normal(12, rows, 2 * hd), normal(13, rows, 2 * hd)
    ang = sc.rope_angles(pos, section, hd, 100.0, restart)
    r = sc.rotate(x, ang, hd, halves)
    assert np.allclose(sc.rotate(r, ang, hd, halves, True), x, atol=1e-12)
    assert np.allclose((r ** 2).sum(), (x ** 2).sum())
    moved = sc.rope_angles(pos + 17, section, hd, 100.0, restart)
    assert np.allclose((r[0, :hd] * sc.rotate(y, ang, hd, halves)[1, :hd]).sum(), (sc.rotate(x, moved, hd, halves)[0, :hd] * sc.rotate(y, moved, hd, halves)[1, :hd]).sum())
    assert ang[0, 0] == pos[0, 0] and np.isclose(ang[0, section[0] - 1], pos[0, 0] * 100.0 ** (-(section[0] - 1) / (section[0] if restart else hd / 2)))


def test_qk_norm_backward_against_differences():
    rows, h, hkv, hd, eps = 5, 2, 1, 6, 1e-3
    t = dict(x=normal(14, rows, (h + hkv) * hd), gq=1 + 0.1 * normal(15, hd), gk=1 + 0.1 * normal(16, hd))
    g = normal(17, rows, (h + hkv) * hd)
    loss = lambda: float((sc.qk_norm(t["x"], t["gq"], t["gk"], h, hkv, eps)[0] * g).sum())
    w, rstd = sc.qk_norm(t["x"], t["gq"], t["gk"], h, hkv, eps)
    grads = dict(zip(("x", "gq", "gk"), sc.qk_norm_backward(t["x"], rstd, t["gq"], t["gk"], h, hkv, g)))
    assert np.allclose((w.reshape(rows, -1, hd)[0, 0] / t["gq"] / t["x"][0, :hd]), rstd[0, 0])
    rng = np.random.default_rng(6)
    for n in t:
        for _ in range(10):
            i = tuple(rng.integers(0, s) for s in t[n].shape)
            was, e = t[n][i], 1e-5
            t[n][i] = was + e
            up = loss()
            t[n][i] = was - e
            down = loss()
            t[n][i] = was
            assert abs((up - down) / (2 * e) - grads[n][i]) <= 1e-7 * (1.0 + abs(grads[n][i])), (n, i)


# ---- refusals: every argument that is not taken, one at a time, on addresses that nothing reads --------------------------------
def A(off=0):
    return 0x10000 + off


def score(**kw):
    from paper_2507_00217_amd import stage as S
    return S.ScoreAttention(**dict(dict(dtype=1, rows=128, n_seq=2, h=4, hkv=2, hd=64, causal=1), **kw))


BAD_SCORE = [dict(dtype=2), dict(rows=0), dict(rows=-1), dict(rows=(1 << 23) + 2), dict(n_seq=0), dict(n_seq=(1 << 20) + 1), dict(n_seq=3), dict(h=0), dict(hkv=0),
             dict(h=3), dict(hd=32), dict(hd=96), dict(causal=2), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(softcap=-1.0),
             dict(softcap=float("nan")), dict(softcap=float("inf")), dict(causal=0, prefix=A()),
             dict(scale=1e-31), dict(softcap=1e-5), dict(scale=1.0, softcap=9e-5)]


@pytest.mark.parametrize("bad", BAD_SCORE)
def test_attention_refuses(bad):
    from paper_2507_00217_amd import stage as S
    L, a = S.lib(), score(**bad)
    m = [A(), 256, A(), 128, A(), 128, A(), 256]
    assert L.stage_kernel_score_attention_fwd(C.byref(a), *m, A(), 0, None) == S.E_INVAL
    assert L.stage_kernel_score_attention_bwd(C.byref(a), *m, A(), A(), 256, A(), 256, A(), 128, A(), 128, A(), 1 << 30, 0, None) == S.E_INVAL
    assert L.stage_kernel_score_attention_bwd_scratch_bytes(C.byref(a)) == 0


def test_attention_refuses_matrices():
    from paper_2507_00217_amd import stage as S
    L, a = S.lib(), score()
    need = L.stage_kernel_score_attention_bwd_scratch_bytes(C.byref(a))
    assert need >= 4 * 128 * 4
    assert L.stage_kernel_score_attention_fwd(None, *[A(), 256, A(), 128, A(), 128, A(), 256], A(), 0, None) == S.E_INVAL
    assert L.stage_kernel_score_attention_bwd_scratch_bytes(None) == 0
    fwd = [A(), 256, A(), 128, A(), 128, A(), 256]
    for i in range(8):
        m = list(fwd)
        m[i] = None if i % 2 == 0 else m[i] - 1
        assert L.stage_kernel_score_attention_fwd(C.byref(a), *m, A(), 0, None) == S.E_INVAL, i
    bwd = fwd + [A(), A(), 256, A(), 256, A(), 128, A(), 128, A(), need]
    for i in [0, 2, 4, 6, 8, 9, 11, 13, 15, 17]:
        m = list(bwd)
        m[i] = None
        assert L.stage_kernel_score_attention_bwd(C.byref(a), *m, 0, None) == S.E_INVAL, i
    for i in [1, 3, 5, 7, 10, 12, 14, 16, 18]:
        m = list(bwd)
        m[i] -= 1
        assert L.stage_kernel_score_attention_bwd(C.byref(a), *m, 0, None) == S.E_INVAL, i
    m = list(bwd)
    m[17] = A(8)                                                         # scratch off its 16 bytes
    assert L.stage_kernel_score_attention_bwd(C.byref(a), *m, 0, None) == S.E_INVAL


def axes(**kw):
    from paper_2507_00217_amd import stage as S
    return S.RopeAxes(**dict(dict(n_axes=2, section=(16, 16), theta=1e4, pos=A(), pos_stride=64), **kw))


BAD_AXES = [dict(n_axes=0), dict(n_axes=5), dict(section=(16, 15)), dict(section=(16, 17)), dict(section=(32, 0)), dict(section=(33, -1)), dict(n_axes=1),
            dict(n_axes=3, section=(16, 16, 0)), dict(section=(2 ** 31 - 1, 2 ** 31 - 1)), dict(halves=2), dict(restart=-1), dict(theta=0.0), dict(theta=-1.0), dict(theta=float("nan")), dict(theta=float("inf")),
            dict(pos=None), dict(pos_stride=63)]


@pytest.mark.parametrize("bad", BAD_AXES)
def test_rotation_refuses_axes(bad):
    from paper_2507_00217_amd import stage as S
    L, a = S.lib(), axes(**bad)
    assert L.stage_kernel_rope_axes(1, 64, 6, 64, C.byref(a), 0, A(), 384, A(), 384, None) == S.E_INVAL
    assert L.stage_kernel_qk_norm_rope_fwd(1, 64, 4, 2, 64, 1e-5, C.byref(a), A(), 384, A(), A(), A(), 384, A(), None) == S.E_INVAL
    assert L.stage_kernel_qk_norm_rope_bwd(1, 64, 4, 2, 64, C.byref(a), A(), 384, A(), A(), A(), A(4096), 384, A(4096), 384, A(), A(64), A(), None) == S.E_INVAL


def test_rotation_and_norm_refuse_the_rest():
    from paper_2507_00217_amd import stage as S
    L, a = S.lib(), axes()
    rope = [1, 64, 6, 64, C.byref(a), 0, A(), 384, A(), 384, None]
    fwd = [1, 64, 4, 2, 64, 1e-5, C.byref(a), A(), 384, A(), A(), A(), 384, A(), None]
    bwd = [1, 64, 4, 2, 64, C.byref(a), A(), 384, A(), A(), A(), A(4096), 384, A(4096), 384, A(), A(64), A(), None]

    def refused(fn, args, at, *values):
        for v in values:
            m = list(args)
            m[at] = v
            assert fn(*m) == S.E_INVAL, (fn, at, v)
    for fn, args, heads in ((L.stage_kernel_rope_axes, rope, 1), (L.stage_kernel_qk_norm_rope_fwd, fwd, 2), (L.stage_kernel_qk_norm_rope_bwd, bwd, 2)):
        refused(fn, args, 0, 2, -1)
        refused(fn, args, 1, 0, -5, (1 << 23) + 1)
        for i in range(heads):
            refused(fn, args, 2 + i, 0, -1, 1 << 16, 2 ** 31 - 1)
        refused(fn, args, 2 + heads, 32, 96, 256)
    refused(L.stage_kernel_rope_axes, rope, 4, None)
    for i in (6, 8):
        refused(L.stage_kernel_rope_axes, rope, i, None, A(8))
    for i in (7, 9):
        refused(L.stage_kernel_rope_axes, rope, i, 376, 385, 392)              # too narrow, off 16 bytes, in place with two strides
    refused(L.stage_kernel_qk_norm_rope_fwd, fwd, 5, -1.0, float("nan"), float("inf"))
    for i in (7, 9, 10, 11):
        refused(L.stage_kernel_qk_norm_rope_fwd, fwd, i, None, A(8))
    for i in (8, 12):
        refused(L.stage_kernel_qk_norm_rope_fwd, fwd, i, 376, 385, 392)
    for i in (6, 9, 10, 11, 13):
        refused(L.stage_kernel_qk_norm_rope_bwd, bwd, i, None, A(8))
    for i in (8, 15, 16, 17):
        refused(L.stage_kernel_qk_norm_rope_bwd, bwd, i, None)
    for i in (7, 12, 14):
        refused(L.stage_kernel_qk_norm_rope_bwd, bwd, i, 376, 385)
    refused(L.stage_kernel_qk_norm_rope_bwd, bwd, 13, A())                     # dx over x
    refused(L.stage_kernel_qk_norm_rope_bwd, bwd, 16, A())                     # one buffer for both weights' gradients
    assert L.stage_kernel_qk_norm_rope_partial_bytes(96) == 0 and L.stage_kernel_qk_norm_rope_partial_bytes(64) > 0
