"""Limits of the shaped-score attention's scalar arguments: the constants that the kernels are handed are fp32 numbers.  Runs without a GPU: refused
calls launch nothing, and what is accepted is asked for its scratch only."""
import ctypes as C

import pytest

from tests.test_score_pins import A, score

# (scale, softcap): the highest coefficient of the tanh polynomial grows with scale (scale / softcap)^8, the others with scale and softcap themselves
BEYOND = [(1e9, 1e5), (1e20, 1e17), (1e30, 1e29), (3e38, 0.0), (2e30, 0.0), (2e30, 1e31), (1.0, 3e38)]
WITHIN = [(1e30, 0.0), (1e30, 1e30), (1e9, 1e9), (1e6, 1e2), (1.0, 1e38), (1e-30, 1e38), (1.0, 1.1e-4), (1e-30, 1e-30)]


@pytest.mark.parametrize("scale,cap", BEYOND)
def test_constants_that_fp32_does_not_hold_are_refused(scale, cap):
    from paper_2507_00217_amd import stage as S
    L, a = S.lib(), score(scale=scale, softcap=cap)
    m = [A(), 256, A(), 128, A(), 128, A(), 256]
    assert L.stage_kernel_score_attention_fwd(C.byref(a), *m, A(), 0, None) == S.E_INVAL
    assert L.stage_kernel_score_attention_bwd(C.byref(a), *m, A(), A(), 256, A(), 256, A(), 128, A(), 128, A(), 1 << 30, 0, None) == S.E_INVAL
    assert L.stage_kernel_score_attention_bwd_scratch_bytes(C.byref(a)) == 0


@pytest.mark.parametrize("scale,cap", WITHIN)
def test_what_they_hold_is_taken(scale, cap):
    from paper_2507_00217_amd import stage as S
    assert S.lib().stage_kernel_score_attention_bwd_scratch_bytes(C.byref(score(scale=scale, softcap=cap))) > 0
