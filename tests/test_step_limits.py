"""Hyperparameters of the AdamW step that fp32, in which it is computed, does not hold.  Runs without a GPU: lists without tensors launch nothing."""
import ctypes as C

import pytest


def adamw(**kw):
    from paper_2507_00217_amd import stage as S
    p = S.AdamW(**dict(dict(dtype=0, grad_dtype=0, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1), **kw))
    return S.lib().stage_kernel_adamw(C.byref(p), 0, None, None, None, None, None, None, None)


@pytest.mark.parametrize("kw", [dict(lr=1e39), dict(weight_decay=1e39), dict(eps=1e39), dict(lr=1.7e308), dict(eps=1e-46), dict(eps=1e-39), dict(eps=5e-324)])
def test_what_fp32_does_not_hold_is_refused(kw):
    """A rate of 1e39 was infinite, and its product with an update of zero NaN; an eps of 1e-46 was zero, and a weight without a gradient 0 / 0."""
    from paper_2507_00217_amd import stage as S
    assert adamw(**kw) == S.E_INVAL


@pytest.mark.parametrize("kw", [{}, dict(lr=0.0), dict(lr=1e38), dict(lr=1e-60), dict(weight_decay=0.0), dict(weight_decay=1e-60), dict(eps=0.0), dict(eps=1e-37), dict(eps=1e38),
                                dict(beta1=0.0, beta2=0.0), dict(beta2=1 - 2.0 ** -53), dict(step=2**31 - 1)])
def test_what_it_holds_is_taken(kw):
    assert adamw(**kw) == 0
