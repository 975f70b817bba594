"""The oracle's rotation (oracle/score_oracle.py) as a complex multiplication: a pair (a, b) is a + ib, turned by exp(i angle).  Runs without a GPU."""
import numpy as np
import pytest

from oracle import score_oracle as sc


@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_is_a_complex_multiplication(halves, inverse):
    rows, heads, hd, section, theta = 7, 3, 16, [3, 4, 1], 1000.0
    rng = np.random.default_rng(5)
    pos, x = rng.integers(-40, 400, (3, rows)), rng.standard_normal((rows, heads * hd))
    pair = np.arange(hd // 2)
    axis = np.repeat(np.arange(3), section)
    turn = np.exp((-1j if inverse else 1j) * pos[axis].T * theta ** (-2.0 * pair / hd))
    v = x.reshape(rows, heads, hd)
    z = (v[..., :hd // 2] + 1j * v[..., hd // 2:] if halves else v[..., 0::2] + 1j * v[..., 1::2]) * turn[:, None, :]
    want = np.concatenate((z.real, z.imag), 2) if halves else np.stack((z.real, z.imag), 3).reshape(rows, heads, hd)
    got = sc.rotate(x, sc.rope_angles(pos, section, hd, theta, 0), hd, halves, inverse)
    assert np.allclose(got, want.reshape(rows, -1), rtol=0, atol=1e-12)
