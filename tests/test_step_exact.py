"""Pins of tests/step_exact.py: it takes what oracle/step_oracle.py gives, rounded, and refuses what is off by more than its bounds.  Runs without a GPU."""
import math

import numpy as np
import pytest
import torch

from oracle import step_oracle as st
from tests.step_exact import E, Rows


def problem(dtype):
    rng = np.random.default_rng(4)
    x = torch.tensor(rng.normal(0, 3, (9, 40))).to(dtype)
    x[1], x[2], x[3, 5], x[4, 7] = -math.inf, math.nan, math.inf, -math.inf
    target = torch.tensor([0, 1, 2, 3, 7, -1, 40, 8, 9])
    w, dh, dl = (torch.tensor(rng.normal(0, 1, 9)).float() for _ in range(3))
    w[8] = dh[8] = dl[8] = 0.0
    n = x.double().numpy()
    scale = float(np.float32(0.7))
    o = st.token_logprob(n, scale, target.numpy())
    g = st.token_logprob_grad(o["all"], o["entropy"], scale, target.numpy(), w.double().numpy(), dh.double().numpy(), dl.double().numpy(), o["stats"][:, 0] == -np.inf)
    f = lambda a: torch.tensor(a).float()
    return Rows(x, 0.7, target, 40), dict(logp=f(o["logp"]), stats=f(o["stats"]), entropy=f(o["entropy"])), torch.tensor(g).float().to(dtype), (w, dh, dl)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_it_takes_the_definition_and_no_more(dtype):
    rows, values, dx, grads = problem(dtype)
    rows.check_values(**values)
    rows.check_grad(dx, *grads)
    for k in values:
        for r in (0, 5, 7):
            wrong = {n: v.clone() for n, v in values.items()}
            at = wrong[k][r] if k != "stats" else wrong[k][r, 1]
            at += 1e-4 if at != 0 or k != "logp" else 1.0
            with pytest.raises(AssertionError):
                rows.check_values(**wrong)
    for r, c, v in ((1, 3, math.nan), (2, 3, 0.0), (3, 0, 0.0), (4, 7, 0.0), (8, 2, 1e-3), (0, 1, None), (7, 8, None)):
        wrong = dx.clone()
        wrong[r, c] = wrong[r, c] * (1 + 2.0 ** (-5 if dtype == torch.bfloat16 else -12)) if v is None else v
        with pytest.raises(AssertionError):
            rows.check_grad(wrong, *grads)
    assert float(rows.e_ln[0]) < 150 * E and float(rows.e_h[0]) < 1500 * E
