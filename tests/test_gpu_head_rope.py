"""Rotary positions on several axes, and the per-head norm of queries and keys with the rotation behind it, against their
definitions in 64 bits.  Elementwise bounds: one rounding of an output, plus what fp32 arithmetic does to a pair (sine and cosine, two
products, the norm's sum): F of the pair's length, 2^-17 with the sine instruction of the bf16 path, 2^-20 in fp32."""
import ctypes as C

import numpy as np
import pytest

from oracle import score_oracle as sc
from paper_2507_00217_amd import synth
from tests.gpu_util import rnd, to_dev, to_np
from tests.score_util import DT, U, close, int_tensor, ptr, wide

pytestmark = pytest.mark.gpu
F = {"fp32": 2.0 ** -20, "bf16": 2.0 ** -17}
SECTIONS = {(1, 64): [32], (1, 128): [64], (2, 64): [16, 16], (2, 128): [23, 41], (3, 64): [8, 12, 12], (3, 128): [16, 24, 24], (4, 64): [7, 1, 13, 11],
            (4, 128): [1, 30, 2, 31]}


def positions(n_axes, rows, seed):
    rng = np.random.default_rng(seed)
    p = rng.integers(0, 3000, (n_axes, rows))
    p[0] = rng.integers(-5, 2 ** 20, rows)                       # far positions, and some before zero
    p[0, 0] = 0
    return p


def axes_of(n_axes, hd, rows, theta, halves, restart, seed=3):
    from paper_2507_00217_amd import stage as S
    pos = positions(n_axes, rows, seed)
    dev = int_tensor(np.concatenate((pos, np.full((n_axes, 3), 2 ** 30)), 1))          # rows of a stride of their own
    sec = SECTIONS[(n_axes, hd)]
    a = S.RopeAxes(n_axes=n_axes, section=tuple(sec), halves=halves, restart=restart, theta=theta, pos=dev.data_ptr(), pos_stride=dev.stride(0))
    return a, dev, sc.rope_angles(pos, sec, hd, np.float32(theta), restart)


def pair_length(x, hd, halves):
    """length of the pair that an element belongs to, at both of its places"""
    v = x.reshape(x.shape[0], -1, hd)
    a, b = (v[..., :hd // 2], v[..., hd // 2:]) if halves else (v[..., 0::2], v[..., 1::2])
    l, out = np.hypot(a, b), np.empty_like(v)
    if halves:
        out[..., :hd // 2] = out[..., hd // 2:] = l
    else:
        out[..., 0::2] = out[..., 1::2] = l
    return out.reshape(x.shape)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("n_axes,restart", [(1, 0), (2, 1), (3, 0), (4, 1)])
@pytest.mark.parametrize("rows,heads", [(1, 1), (37, 5), (130, 20)])
def test_rope_axes(dtype, hd, halves, n_axes, restart, rows, heads):
    import torch
    from paper_2507_00217_amd import stage as S
    x = rnd(synth.normal(51, 1, (rows, heads * hd)), dtype)
    axes, keep, ang = axes_of(n_axes, hd, rows, 1e6 if restart else 1e4, halves, restart)
    for inverse in (0, 1):
        ref = sc.rotate(x, ang, hd, halves, bool(inverse))
        bound = U[dtype] * np.abs(ref) + F[dtype] * pair_length(x.astype(np.float64), hd, halves)
        xd, y = wide(x, dtype, 16), wide(np.full(x.shape, np.nan, np.float32), dtype, 8)
        assert S.lib().stage_kernel_rope_axes(DT[dtype], rows, heads, hd, C.byref(axes), inverse, ptr(xd), xd.stride(0), ptr(y), y.stride(0), None) == 0
        torch.cuda.synchronize()
        close("y", to_np(y[:, :heads * hd]), ref, bound)
        assert bool(torch.isnan(y[:, heads * hd:].float()).all())
        first = y.clone()
        assert S.lib().stage_kernel_rope_axes(DT[dtype], rows, heads, hd, C.byref(axes), inverse, ptr(xd), xd.stride(0), ptr(xd), xd.stride(0), None) == 0
        torch.cuda.synchronize()
        assert torch.equal(first[:, :heads * hd], xd[:, :heads * hd])          # in place: the same bits
        assert bool(torch.isnan(xd[:, heads * hd:].float()).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
def test_one_axis_is_the_engines_rotation(dtype, hd):
    """Positions 0, 1, 2, ... on one axis and adjacent pairs: what stage_kernel_rope does with its table, to a rounding."""
    import torch
    from paper_2507_00217_amd import stage as S
    L, s, heads = S.lib(), 300, 3
    x = rnd(synth.normal(52, 1, (s, heads * hd)), dtype)
    pos = torch.arange(s, dtype=torch.int32, device="cuda:0")
    axes = S.RopeAxes(n_axes=1, section=(hd // 2,), theta=1e4, pos=pos.data_ptr(), pos_stride=s)
    a, b, table = to_dev(x, dtype), to_dev(x, dtype), torch.empty(s, hd // 2, 2, device="cuda:0")
    assert L.stage_kernel_rope_table(s, hd, C.c_float(1e4), C.c_void_p(ptr(table)), None) == 0
    assert L.stage_kernel_rope(DT[dtype], 1, s, heads, hd, 0, C.c_void_p(ptr(a)), C.c_int64(heads * hd), C.c_void_p(ptr(table)), None) == 0
    assert L.stage_kernel_rope_axes(DT[dtype], s, heads, hd, C.byref(axes), 0, ptr(b), heads * hd, ptr(b), heads * hd, None) == 0
    torch.cuda.synchronize()
    ref = to_np(a)
    close("y", to_np(b), ref, 2 * U[dtype] * np.abs(ref) + 2 * F[dtype] * pair_length(x.astype(np.float64), hd, 0))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("n_axes,rows,h,hkv", [(0, 70, 3, 1), (1, 1, 1, 1), (1, 333, 8, 2), (3, 130, 12, 4), (1, 2100, 1, 1)])
def test_qk_norm_rope(dtype, hd, halves, n_axes, rows, h, hkv):
    """Forward and backward; dgamma is added to what is there; columns behind the heads stay; dx in the place of dy is the same."""
    import torch
    from paper_2507_00217_amd import stage as S
    L, n, eps = S.lib(), (h + hkv) * hd, 1e-5
    x = rnd(synth.normal(61, 1, (rows, n), std=1.7), dtype)
    x[0, :hd] = 0.0                                                  # a head of zeros: rstd = eps^(-1/2)
    gq, gk = (rnd(synth.normal(61, i, (hd,), mean=1.0, std=0.2), dtype) for i in (2, 3))
    dy = rnd(synth.normal(61, 4, (rows, n)), dtype)
    dg0 = synth.normal(61, 5, (2, hd))
    if n_axes:
        axes, keep, ang = axes_of(n_axes, hd, rows, 1e4, halves, 0)
        ref_axes = C.byref(axes)
    else:
        ref_axes, ang = None, np.zeros((rows, hd // 2))
    w, rstd_ref = sc.qk_norm(x, gq, gk, h, hkv, eps)
    xd, dyd, gqd, gkd, dg = wide(x, dtype, 8), wide(dy, dtype, 16), to_dev(gq, dtype), to_dev(gk, dtype), to_dev(dg0, "fp32")
    y, dx = wide(np.full(x.shape, np.nan, np.float32), dtype, 24), wide(np.full(x.shape, np.nan, np.float32), dtype, 8)
    rstd = torch.full((rows, h + hkv), float("nan"), device="cuda:0")
    fwd = lambda out, keep_rstd=True: L.stage_kernel_qk_norm_rope_fwd(DT[dtype], rows, h, hkv, hd, eps, ref_axes, ptr(xd), xd.stride(0), ptr(gqd), ptr(gkd),
                                                                      ptr(out), out.stride(0), ptr(rstd) if keep_rstd else None, None)
    assert fwd(y) == 0
    torch.cuda.synchronize()
    ref = sc.rotate(w, ang, hd, halves)
    close("y", to_np(y[:, :n]), ref, U[dtype] * np.abs(ref) + F[dtype] * pair_length(w, hd, halves))
    close("rstd", to_np(rstd), rstd_ref, F["fp32"] * rstd_ref)
    assert bool(torch.isnan(y[:, n:].float()).all())
    part = torch.full((L.stage_kernel_qk_norm_rope_partial_bytes(hd) // 4,), float("nan"), device="cuda:0")
    bwd = lambda dyt, dxt, dgt: L.stage_kernel_qk_norm_rope_bwd(DT[dtype], rows, h, hkv, hd, ref_axes, ptr(xd), xd.stride(0), ptr(rstd), ptr(gqd), ptr(gkd), ptr(dyt),
                                                                dyt.stride(0), ptr(dxt), dxt.stride(0), ptr(dgt[0]), ptr(dgt[1]), ptr(part), None)
    assert bwd(dyd, dx, dg) == 0
    torch.cuda.synchronize()
    r32 = to_np(rstd)
    g = sc.rotate(dy, ang, hd, halves, True)
    dx_ref, dgq_ref, dgk_ref = sc.qk_norm_backward(x, r32, gq, gk, h, hkv, g)
    glen, nlen = pair_length(g, hd, halves).reshape(rows, -1, hd), np.abs(x.astype(np.float64)).reshape(rows, -1, hd) * r32[..., None]
    gam = np.concatenate((np.repeat(np.abs(gq)[None], h, 0), np.repeat(np.abs(gk)[None], hkv, 0)))
    mag = r32[..., None] * (glen * gam + nlen * (glen * gam * nlen).mean(-1, keepdims=True))
    close("dx", to_np(dx[:, :n]), dx_ref, U[dtype] * np.abs(dx_ref) + F[dtype] * mag.reshape(rows, n))
    terms = (glen * nlen).sum(0)
    for i, (got, want, t, m) in enumerate(((dg[0], dgq_ref, terms[:h].sum(0), 1), (dg[1], dgk_ref, terms[h:].sum(0), 1))):
        close("dgamma", to_np(got), want + dg0[i], F[dtype] * t + U["fp32"] * np.abs(dg0[i]))
    assert bool(torch.isnan(dx[:, n:].float()).all())
    # in place, and again: the same bits
    dg2 = to_dev(dg0, "fp32")
    assert bwd(dyd, dyd, dg2) == 0
    torch.cuda.synchronize()
    assert torch.equal(dyd[:, :n], dx[:, :n]) and torch.equal(dg, dg2)
    assert fwd(xd, False) == 0
    torch.cuda.synchronize()
    assert torch.equal(xd[:, :n], y[:, :n]) and bool(torch.isnan(xd[:, n:].float()).all())


@pytest.mark.parametrize("dtype,hd,per_step", [("fp32", 128, 2), ("fp32", 64, 4), ("bf16", 128, 4), ("bf16", 64, 8)])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6, 7, 8, 9, 11])
def test_shares_of_a_row_agree_bitwise(dtype, hd, per_step, steps):
    """With rows enough to fill the chip a wavefront takes several steps of a row's heads (a row is `steps` of them, the last one cut short), with a
    hundred rows one: the same bits either way, forward and (whose shares do not depend on the rows) backward."""
    import torch
    from paper_2507_00217_amd import stage as S
    L, rows, few = S.lib(), 4103, 100
    heads = steps * per_step - (1 if steps > 1 else 0)
    h, hkv = max(1, heads - 1 - steps // 3), heads - max(1, heads - 1 - steps // 3)
    n, g = heads * hd, torch.Generator(device="cuda:0").manual_seed(7)
    td = torch.float32 if dtype == "fp32" else torch.bfloat16
    x, dy = (torch.randn(rows, n, generator=g, device="cuda:0").to(td) for _ in range(2))
    gam = (1 + 0.1 * torch.randn(2, hd, generator=g, device="cuda:0")).to(td)
    axes, keep, _ = axes_of(2, hd, rows, 1e4, steps % 2, 0)
    part = torch.empty(L.stage_kernel_qk_norm_rope_partial_bytes(hd), dtype=torch.uint8, device="cuda:0")

    def run(r):
        y, z, dx = (torch.full((r, n), float("nan"), device="cuda:0").to(td) for _ in range(3))
        rstd, dg = torch.full((r, heads), float("nan"), device="cuda:0"), torch.zeros(2, hd, device="cuda:0")
        assert L.stage_kernel_qk_norm_rope_fwd(DT[dtype], r, h, hkv, hd, 1e-5, C.byref(axes), ptr(x), n, ptr(gam[0]), ptr(gam[1]), ptr(y), n, ptr(rstd), None) == 0
        assert L.stage_kernel_rope_axes(DT[dtype], r, heads, hd, C.byref(axes), 1, ptr(x), n, ptr(z), n, None) == 0
        assert L.stage_kernel_qk_norm_rope_bwd(DT[dtype], r, h, hkv, hd, C.byref(axes), ptr(x), n, ptr(rstd), ptr(gam[0]), ptr(gam[1]), ptr(dy), n, ptr(dx), n,
                                               ptr(dg[0]), ptr(dg[1]), ptr(part), None) == 0
        torch.cuda.synchronize()
        return y, z, rstd, dx, dg
    many, short = run(rows), run(few)
    for a, b in zip(many[:4], short[:4]):
        assert bool(torch.isfinite(a.float()).all()) and torch.equal(a[:few], b)
    # the weights' gradients of all rows, from the kernel's own rstd, in 64 bits
    f = lambda t: t.double().cpu().numpy()
    ang = sc.rope_angles(keep.cpu().numpy()[:, :rows], SECTIONS[(2, hd)], hd, np.float32(1e4), 0)
    gr = sc.rotate(f(dy), ang, hd, steps % 2, True)
    _, dgq, dgk = sc.qk_norm_backward(f(x), f(many[2]), f(gam[0]), f(gam[1]), h, hkv, gr)
    terms = (pair_length(gr, hd, steps % 2).reshape(rows, heads, hd) * (np.abs(f(x)).reshape(rows, heads, hd) * f(many[2])[..., None])).sum(0)
    close("dgq", to_np(many[4][0]), dgq, F[dtype] * terms[:h].sum(0))
    close("dgk", to_np(many[4][1]), dgk, F[dtype] * terms[h:].sum(0))
